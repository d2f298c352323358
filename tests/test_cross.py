"""Rotary positions with several axes, written to a cache or to dense states, and HCCS attention to states of another length.

Codes and integer outputs are compared for equality, float outputs with the tolerances of test_cache.compare: one product
of an exact integer with a rounded factor.
"""
import ctypes
import math

import numpy as np
import pytest

from oracle import hccs_cache_oracle as orc
from test_cache import _f, _theta, _torch_type, _values, compare

TYPES = ("bf16", "f16", "f32")


# ------------------------------------------------------------------------------------------- host only
@pytest.fixture(scope="module")
def binding():
    from paper_2604_02292_b200 import build
    build.build()
    from paper_2604_02292_b200 import binding as b
    return b


@pytest.mark.parametrize("pairs", [(16, 24, 24), (64,), (1, 62, 1), (16, 16), (0, 8, 8), (5, 0, 3, 24), (24, 20, 20), (7, 9)])
@pytest.mark.parametrize("restart", [False, True])
def test_rope_axes_by_their_definition(binding, pairs, restart):
    b = binding
    half = sum(pairs)
    sections = [x for x, n in enumerate(pairs) for _ in range(n)]
    left, turns, x = list(pairs), [], 0
    while len(turns) < half:
        if left[x]:
            turns.append(x)
            left[x] -= 1
        x = (x + 1) % len(pairs)
    for order, want in ((b.HCCS_AXES_SECTIONS, sections), (b.HCCS_AXES_TURNS, turns)):
        r = b.hccs_rope_axes(2 * half, pairs, base=500.0, interleaved=True, order=order, restart=restart, kind=b.HCCS_ROPE_LINEAR, factor=3.0)
        assert r.num_axes == len(pairs) and r.rope.rot_dim == 2 * half and r.rope.interleaved == 1 and r.rope.scale == 1.0
        assert list(r.axis)[:half] == want and not any(list(r.axis)[half:])
        seen = [0] * len(pairs)
        for i, a in enumerate(want):
            f = 500.0 ** (-seen[a] / pairs[a]) if restart else 500.0 ** (-i / half)
            assert math.isclose(r.rope.freq[i], f / 3, rel_tol=1e-13), (i, a)
            seen[a] += 1
    one = b.hccs_rope_frequencies(2 * half, 500.0)
    r = b.hccs_rope_axes(2 * half, (half,), base=500.0, restart=restart)
    assert list(r.rope.freq) == list(one.freq)             # one axis is the plain call


def test_rope_axes_refusals(binding):
    b = binding
    for kw in (dict(rot_dim=0, pairs=(0,)), dict(rot_dim=63, pairs=(31,)), dict(pairs=(16, 17)), dict(pairs=(16, 15)), dict(pairs=(-1, 33)),
               dict(pairs=()), dict(pairs=(8, 8, 8, 4, 4)), dict(order=2), dict(order=-1), dict(base=1.0), dict(kind=9),
               dict(pairs=(1, 31), restart=True, kind=2, factor=2.0)):
        args = dict(rot_dim=64, pairs=(16, 16))
        args.update(kw)
        with pytest.raises(b.HccsError) as ei:
            b.hccs_rope_axes(**args)
        assert ei.value.status == b.HCCS_ERR_INVALID_ARG, kw
    lib = b.raw()
    assert lib.hccs_rope_axes(None, 64, 0, 1e4, None, ctypes.byref((ctypes.c_int32 * 1)(32)), 1, 0, 0) == b.HCCS_ERR_INVALID_ARG
    assert lib.hccs_rope_axes(ctypes.byref(b.RopeAxes()), 64, 0, 1e4, None, None, 1, 0, 0) == b.HCCS_ERR_INVALID_ARG
    for args in (([1.0], [0, 1]), ([1.0], [4]), ([1.0], [-1]), ([1.0] * 65, [0] * 65)):
        with pytest.raises(ValueError):
            b.RopeAxes(*args)
    with pytest.raises(ValueError):
        b.RopeAxes([1.0, 1.0], [0, 1], num_axes=1)


def test_write_refusals_without_a_gpu(binding):
    """Argument checks that need no context come first; what passes them all ends at the NULL context."""
    b, lib = binding, binding.raw()
    P = 4096                                               # an aligned address that is never read
    two = _f(0.1, 0.1)
    good = b.RopeAxes([1.0] * 8, [0, 1, 2, 0, 1, 2, 0, 1])
    bad_axis, no_axes, many = (b.RopeAxes([1.0] * 8, [0, 1, 2, 0, 1, 2, 0, 1]) for _ in range(3))
    bad_axis.axis[7] = 3
    no_axes.num_axes = 0
    many.num_axes = 5

    def call(paged, **kw):
        a = dict(q=P, k=P, v=P, type=b.HCCS_F32, qs=64, ks=64, vs=64, pos=P, slots=P, rope=good, q_step=two, k_step=two, v_step=two, q8=P,
                 k8=P, v8=P, T=6, L=3, Hq=2, Hkv=2, d=64, pages=4, size=16)
        a.update(kw)
        ptr = {n: (a[n].ctypes.data if a[n] is not None else None) for n in ("q_step", "k_step", "v_step")}
        head = (None, a["q"], a["k"], a["v"], a["type"], a["qs"], a["ks"], a["vs"], a["pos"], 6, 1)
        rope = ctypes.byref(a["rope"]) if a["rope"] else None
        tail = (rope, ptr["q_step"], ptr["k_step"], ptr["v_step"], a["q8"], a["k8"], a["v8"], a["T"])
        if paged:
            return lib.hccs_cache_write_axes(*head, a["slots"], *tail, a["Hq"], a["Hkv"], a["d"], a["pages"], a["size"], None)
        return lib.hccs_states_write(*head, *tail, a["L"], a["Hq"], a["Hkv"], a["d"], None)
    I, U = b.HCCS_ERR_INVALID_ARG, b.HCCS_ERR_UNSUPPORTED
    for paged in (True, False):
        assert call(paged) == I                            # the NULL context
        for kw in (dict(T=-1), dict(type=0), dict(type=9), dict(k=None), dict(v=None), dict(Hkv=0), dict(Hkv=257), dict(Hq=0), dict(Hq=257),
                   dict(q_step=None), dict(k_step=_f(0.1, 0.0)), dict(v_step=_f(0.1, np.nan)), dict(rope=bad_axis), dict(rope=no_axes),
                   dict(rope=many), dict(rope=b.RopeAxes([1.0] * 33, [0] * 33)), dict(rope=b.RopeAxes([np.inf], [0])), dict(pos=None),
                   dict(q8=None), dict(k8=None), dict(v8=None)):
            assert call(paged, **kw) == I, kw
        for kw in (dict(d=32), dict(q=P + 8), dict(k=P + 4), dict(q8=P + 1), dict(k8=P + 8), dict(v8=P + 8), dict(qs=65), dict(vs=67),
                   dict(type=b.HCCS_BF16, qs=68)):
            assert call(paged, **kw) == U, kw
    for kw in (dict(slots=None), dict(size=24), dict(pages=0)):
        assert call(True, **kw) == I, kw
    for kw in (dict(L=0), dict(L=-3), dict(L=4), dict(L=7)):
        assert call(False, **kw) == I, kw


def test_cross_refusals_without_a_gpu(binding):
    b, lib = binding, binding.raw()
    P = 4096
    I, U = b.HCCS_ERR_INVALID_ARG, b.HCCS_ERR_UNSUPPORTED

    def call(**kw):
        a = dict(Q=P, K=P, V=P, ks=128, vs=128, qs=P, k0=P, kl=P, kr=None, mult=np.array([100, 100], np.int32), shift=20, scale=_f(1, 1),
                 O=P, type=b.HCCS_F32, T=3, S=50, B=2, Hq=2, Hkv=2, d=64, mq=2, mkv=40, flags=0)
        a.update(kw)
        return lib.hccs_attention_cross(None, a["Q"], a["K"], a["V"], a["ks"], a["vs"], a["qs"], a["k0"], a["kl"], a["kr"],
                                        a["mult"].ctypes.data if a["mult"] is not None else None, a["shift"],
                                        a["scale"].ctypes.data if a["scale"] is not None else None, a["O"], a["type"], a["T"], a["S"], a["B"],
                                        a["Hq"], a["Hkv"], a["d"], a["mq"], a["mkv"], a["flags"], None)
    assert call() == I                                     # the NULL context
    for kw in (dict(T=-1), dict(S=-1), dict(B=-1), dict(mq=-1), dict(mkv=-1), dict(flags=1), dict(flags=4), dict(flags=10), dict(type=7),
               dict(scale=None), dict(type=b.HCCS_I32), dict(type=b.HCCS_I32, scale=None, flags=b.HCCS_RECIP_REAL),
               dict(scale=_f(1, np.inf)), dict(mult=None), dict(Hq=3), dict(Hq=0), dict(Hkv=0), dict(Hkv=-1), dict(shift=0), dict(shift=25),
               dict(mult=np.array([-1, 0], np.int32)), dict(mult=np.array([1 << 13, 0], np.int32)), dict(Q=None), dict(K=None), dict(V=None),
               dict(qs=None), dict(k0=None), dict(kl=None), dict(O=None), dict(ks=112), dict(vs=0), dict(ks=-128)):
        assert call(**kw) == I, kw
    for kw in (dict(d=80), dict(B=65536), dict(mkv=131073), dict(Hq=258), dict(shift=5), dict(Q=P + 1), dict(K=P + 8), dict(V=P + 8),
               dict(O=P + 4), dict(kr=P + 4), dict(ks=136), dict(vs=1 << 36), dict(mq=(1 << 30) + 1)):
        assert call(**kw) == U, kw


def test_oracle_of_cross_attention_agrees_with_that_of_the_cache():
    """Queries whose keys are all before them: the same states in pages, or in a row."""
    rng = np.random.default_rng(11)
    n, d, hq, hkv = 48, 64, 4, 2
    q = rng.integers(-64, 64, (3, hq, d), dtype=np.int8)
    k, v = (rng.integers(-64, 64, (5, hkv, 16, d), dtype=np.int8) for _ in range(2))
    table = np.array([[3, 1, 4]])
    theta, mult = _theta(rng, hq, n, False), [2000] * hq
    seq = [orc.sequence(p, table[0], n) for p in (k, v)]
    for t in range(3):
        want = orc.attend(q[t:t + 1], k, v, table, [0, 1], [n], theta, mult, 20)
        got = orc.cross(q[t:t + 1], *seq, [0, 1], [0], [n], theta, mult, 20)
        sliced = orc.cross(q[t:t + 1], *seq, [0, 1], [0], [n], theta, mult, 20, [[10, 31]])
        shifted = orc.cross(q[t:t + 1], *seq, [0, 1], [10], [21], theta, mult, 20)
        for a, c in zip(want, got):
            assert (a == c).all()
        for a, c in zip(sliced, shifted):
            assert (a == c).all()


# ------------------------------------------------------------------------------------------- rotary positions with several axes
def _tokens(rng, T, hq, hkv, d, dtype):
    import torch
    x = torch.from_numpy(rng.standard_normal((T, (hq + 2 * hkv) * d + 16)).astype(np.float32)).to("cuda", _torch_type(dtype))
    return [x[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv))]


WRITES = [  # hq, hkv, d, pairs, order, restart, interleaved, T
    (4, 2, 64, (8, 12, 12), 0, False, False, 1), (4, 2, 128, (24, 20, 20), 1, False, False, 37), (3, 3, 64, (8, 8), 0, True, True, 50),
    (5, 1, 128, (16, 16, 16, 16), 1, True, True, 33), (2, 2, 64, (3, 7), 0, False, False, 20), (8, 2, 128, (1, 1, 1), 1, False, True, 19),
    (6, 3, 64, (9, 2, 1), 0, True, False, 23), (7, 7, 128, (48,), 0, False, False, 40), (16, 4, 64, (1, 31), 0, False, True, 300)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv,d,pairs,order,restart,interleaved,T", WRITES)
def test_cache_write_axes(hccs, dtype, hq, hkv, d, pairs, order, restart, interleaved, T):
    import torch
    rng = np.random.default_rng(hq * 1000 + d + T)
    page = 16
    pages = -(-T // page) + 2
    q, k, v = _tokens(rng, T, hq, hkv, d, dtype)
    pos = rng.integers(-50, 131072, (len(pairs), T)).astype(np.int32)
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    if T > 3:
        slots[2] = -1
    steps = [rng.uniform(0.005, 0.05, n).astype(np.float32) for n in (hq, hkv, hkv)]
    steps[0][0] = 0.03125                                  # a power of two: exact ties
    rope = hccs.hccs_rope_axes(2 * sum(pairs), pairs, interleaved=interleaved, order=order, restart=restart)
    rope.rope.scale = 1.0 if T % 2 else 1.23
    half = sum(pairs)
    freq, axis, scale = list(rope.rope.freq)[:half], list(rope.axis)[:half], rope.rope.scale
    kp, vp = (rng.integers(-128, 128, (pages, hkv, page, d), dtype=np.int8) for _ in range(2))
    xq, xk, xv = (t.float().cpu().numpy() for t in (q, k, v))
    want_q = orc.quantise(orc.rotate_axes(xq, pos, freq, axis, interleaved, scale), steps[0])
    want_k = orc.write(kp, orc.quantise(orc.rotate_axes(xk, pos, freq, axis, interleaved, scale), steps[1]), slots)
    want_v = orc.write(vp, orc.quantise(xv, steps[2]), slots)
    ctx = hccs.Context(0)
    for positions in (torch.from_numpy(pos).cuda(), torch.from_numpy(np.ascontiguousarray(pos.T)).cuda().t()):       # [axes,T] and [T,axes]
        q8 = torch.full((T, hq, d), 99, dtype=torch.int8, device="cuda")
        dk, dv = torch.from_numpy(kp).cuda(), torch.from_numpy(vp).cuda()
        ctx.hccs_cache_write_axes(q, k, v, q8, dk, dv, positions, torch.from_numpy(slots).cuda(), *steps, rope=rope)
        assert ctx.hccs_device_status() == 0
        for name, got, want in (("q", q8, want_q), ("k", dk, want_k), ("v", dv, want_v)):
            assert (got.cpu().numpy() == want).all(), name
    if len(pairs) == 1:                                    # one axis: the plain call
        q9, dk9, dv9 = torch.empty_like(q8), torch.from_numpy(kp).cuda(), torch.from_numpy(vp).cuda()
        ctx.hccs_cache_write(q, k, v, q9, dk9, dv9, torch.from_numpy(pos[0]).cuda(), torch.from_numpy(slots).cuda(), *steps, rope=rope.rope)
        assert torch.equal(q9, q8) and torch.equal(dk9, dk) and torch.equal(dv9, dv)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("batch", [1, 3])
@pytest.mark.parametrize("hq,hkv,d,pairs,order,restart,interleaved,T", WRITES)
def test_states_write(hccs, dtype, batch, hq, hkv, d, pairs, order, restart, interleaved, T):
    """Both layouts, with and without queries, with and without rotation; what lies around the outputs stays."""
    import torch
    rng = np.random.default_rng(hq * 1000 + d + T + batch)
    T = min(T, 60)
    n = T * batch
    q, k, v = _tokens(rng, n, hq, hkv, d, dtype)
    pos = rng.integers(0, 4096, (len(pairs), n)).astype(np.int32)
    steps = [rng.uniform(0.005, 0.05, m).astype(np.float32) for m in (hq, hkv, hkv)]
    steps[1][0] = 2.0 ** -5
    rope = hccs.hccs_rope_axes(2 * sum(pairs), pairs, interleaved=interleaved, order=order, restart=restart)
    half = sum(pairs)
    freq, axis = list(rope.rope.freq)[:half], list(rope.axis)[:half]
    xq, xk, xv = (t.float().cpu().numpy() for t in (q, k, v))
    turned = [orc.quantise(orc.rotate_axes(x, pos, freq, axis, interleaved, 1.0), s) for x, s in ((xq, steps[0]), (xk, steps[1]))]
    plain = [orc.quantise(x, s) for x, s in ((xq, steps[0]), (xk, steps[1]), (xv, steps[2]))]
    ctx = hccs.Context(0)
    positions = torch.from_numpy(pos).cuda()
    for heads_first in (False, True):
        def out(heads):
            flat = torch.full((n * heads * d + 64,), 77, dtype=torch.int8, device="cuda")
            shape = (batch, heads, T, d) if heads_first else (n, heads, d)
            return flat, flat[32:-32].view(shape)

        def tokens_first(t):
            return (t.transpose(1, 2).reshape(n, -1, d) if heads_first else t).cpu().numpy()
        for with_q, with_kv, turn in ((True, True, True), (True, False, True), (False, True, True), (True, True, False)):
            fq, q8 = out(hq)
            fk, k8 = out(hkv)
            fv, v8 = out(hkv)
            ctx.hccs_states_write(q if with_q else None, k if with_kv else None, v if with_kv else None, q8, k8, v8,
                                  positions if turn else None, *steps, rope=rope if turn else None)
            assert ctx.hccs_device_status() == 0
            want = (turned if turn else plain[:2]) + plain[2:]
            for name, flat, got, w, there in (("q", fq, q8, want[0], with_q), ("k", fk, k8, want[1], with_kv), ("v", fv, v8, want[2], with_kv)):
                assert (tokens_first(got) == (w if there else 77)).all(), name
                assert (flat[:32] == 77).all() and (flat[-32:] == 77).all(), name
    ctx.close()


@pytest.mark.gpu
def test_write_axes_of_far_positions_infinities_and_nan(hccs):
    """Angles beyond 2^24 radians on one axis alone, values that are none: the pair's own axis decides."""
    import torch
    rng = np.random.default_rng(3)
    d, T, hq = 64, 40, 3
    x = rng.standard_normal((T, hq, d)).astype(np.float32)
    x[0, 0, 3], x[1, 1, 40], x[2, 2, ::5] = np.nan, np.inf, -np.inf
    freq = [1.0] * 8 + [1000.0 ** (-i / 24) for i in range(24)]
    axis = [1] * 8 + [0] * 24
    pos = np.stack([np.arange(T), rng.integers(-2**31, 2**31 - 1, T)]).astype(np.int32)
    step = np.array([0.03, 0.03125, 0.01], np.float32)
    ctx = hccs.Context(0)
    q8 = torch.empty((T, hq, d), dtype=torch.int8, device="cuda")
    ctx.hccs_states_write(torch.from_numpy(x).cuda(), None, None, q8, None, None, torch.from_numpy(pos).cuda(), step, None, None,
                          rope=hccs.RopeAxes(freq, axis))
    assert (q8.cpu().numpy() == orc.quantise(orc.rotate_axes(x, pos, freq, axis, False, 1.0), step)).all()
    ctx.close()


@pytest.mark.gpu
def test_write_refusals_of_the_binding(hccs):
    import torch
    ctx = hccs.Context(0)
    dev = "cuda"
    q, k = torch.zeros((6, 4, 64), device=dev), torch.zeros((6, 2, 64), device=dev)
    q8, k8, v8 = (torch.zeros((6, h, 64), dtype=torch.int8, device=dev) for h in (4, 2, 2))
    pos = torch.zeros((3, 6), dtype=torch.int32, device=dev)
    rope = hccs.hccs_rope_axes(64, (8, 12, 12))
    steps = [np.full(h, 0.1, np.float32) for h in (4, 2, 2)]

    def call(**kw):
        a = dict(q=q, k=k, v=k, q8=q8, k8=k8, v8=v8, pos=pos, rope=rope)
        a.update(kw)
        ctx.hccs_states_write(a["q"], a["k"], a["v"], a["q8"], a["k8"], a["v8"], a["pos"], *steps, rope=a["rope"])
    call()
    for kw in (dict(pos=pos[:2]), dict(pos=pos[0]), dict(pos=pos[:, :5]), dict(pos=pos.float()), dict(pos=pos.long()), dict(pos=pos.cpu()),
               dict(q8=q8[:5]), dict(k8=k8.float()), dict(v8=v8.cpu()), dict(q=None, k=None, v=None), dict(v=None), dict(v=k.half()),
               dict(q8=torch.zeros((2, 4, 2, 64), dtype=torch.int8, device=dev)), dict(k8=torch.zeros((2, 2, 3, 64), dtype=torch.int8, device=dev))):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(hccs.HccsError):
        call(pos=None)
    # nothing to do
    none = torch.zeros((0, 4, 64), device=dev)
    ctx.hccs_states_write(none, None, None, q8[:0], None, None, None, steps[0], None, None)
    ctx.close()


# ------------------------------------------------------------------------------------------- cross attention
def cross(pkg, ctx, rng, q_lens, k_lens, hq, hkv, d, norm="real", dtype="f32", ranges=None, wide=False, shift=20, mult=None, spread=24.0,
          fused=False, share=None, gap=3, n_design=None, theta=None, q=None, kv=None, max_q=None, check=True, stream=None):
    """One call and its comparison with the oracle.  gap: states between the sequences' own; share: sequence whose states are read."""
    import torch
    T = sum(q_lens)
    start = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
    k_start, at = [], gap
    for b, n in enumerate(k_lens):
        if share and share[b] != b:
            k_start.append(k_start[share[b]])
        else:
            k_start.append(at)
            at += n + gap
    S = at
    kv = rng.integers(-128, 128, (S, 2 * hkv, d), dtype=np.int8) if kv is None else kv
    q = rng.integers(-128, 128, (T, hq, d), dtype=np.int8) if q is None else q
    n = n_design or max(max(k_lens), 1)
    theta = _theta(rng, hq, n, wide) if theta is None else theta
    if mult is None:
        sigma = 74.0 ** 2 * math.sqrt(d)
        mult = np.array([min(8191, (1 << (shift - 1)) - 1, int(spread * rng.uniform(0.3, 1.5) / sigma * (1 << shift))) for _ in range(hq)], np.int32)
    (ctx.hccs_params_upload_wide if wide else ctx.hccs_params_upload)(theta, n)
    scale = rng.uniform(0.01, 0.05, hq).astype(np.float32)
    dev = "cuda"
    out = torch.full((T + 2, hq, d), 77, dtype=_torch_type(dtype), device=dev)         # two rows behind the last sequence
    Q = torch.full((T + 2, hq, d), 3, dtype=torch.int8, device=dev)
    Q[:T] = torch.from_numpy(q).to(dev)
    states = torch.from_numpy(kv).to(dev)
    K, V = states[:, :hkv], states[:, hkv:]
    if not fused:
        K, V = K.contiguous(), V.contiguous()
    R = None
    if ranges is not None:
        R = torch.zeros((T + 2, 2), dtype=torch.int32, device=dev)
        R[:T] = torch.from_numpy(np.asarray(ranges, np.int32).reshape(T, 2)).to(dev)
    args = (Q, K, V, torch.from_numpy(start).to(dev), torch.tensor(k_start, dtype=torch.int32, device=dev),
            torch.tensor(k_lens, dtype=torch.int32, device=dev), out, mult, shift)
    flags = {"real": pkg.HCCS_RECIP_REAL, "div": 0, "clb": pkg.HCCS_RECIP_CLB}[norm]
    kw = dict(max_q=max_q or max(max(q_lens), 1), max_kv=max(max(k_lens), 1), key_range=R, out_scale=None if dtype == "i32" else scale, flags=flags)
    ctx.hccs_attention_cross(*args, **kw)
    torch.cuda.synchronize()
    assert (_values(out[T:]) == 77).all(), "rows behind the last sequence were written"
    if check:
        num, zs, cnt = orc.cross(q, kv[:, :hkv], kv[:, hkv:], start, k_start, k_lens, theta, mult, shift, ranges)
        compare(out[:T], num, zs, cnt, norm, dtype, scale)
        assert ctx.hccs_device_status() == 0
    return out, (args, kw, theta)


@pytest.fixture
def ctx(hccs):
    c = hccs.Context(0)
    yield c
    c.close()


# single queries, few rows: lengths around tiles of 32 keys, heads in groups of every kind
@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", [(1, 1, 64), (3, 3, 128), (8, 2, 64), (7, 1, 128), (16, 1, 64), (12, 1, 128), (40, 2, 128)])
@pytest.mark.parametrize("norm,dtype", [("div", "i32"), ("clb", "i32"), ("real", "f32"), ("real", "bf16"), ("div", "f16"), ("clb", "bf16")])
def test_single_queries(hccs, ctx, hq, hkv, d, norm, dtype):
    rng = np.random.default_rng(hq + d)
    cross(hccs, ctx, rng, [1, 1, 0, 1, 1, 1], [1, 31, 7, 0, 64, 77], hq, hkv, d, norm, dtype, fused=hq % 2 == 0)
    cross(hccs, ctx, rng, [1, 1], [333, 2], hq, hkv, d, norm, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,queries", [(1, 1, 64, 16), (2, 2, 128, 9), (4, 2, 64, 5), (3, 1, 128, 5), (8, 2, 128, 4), (5, 1, 64, 3), (8, 1, 64, 2)])
@pytest.mark.parametrize("norm,dtype", [("div", "i32"), ("real", "f32"), ("real", "f16")])
def test_few_rows(hccs, ctx, hq, hkv, d, queries, norm, dtype):
    """Up to sixteen (query, head) rows of a kv head."""
    rng = np.random.default_rng(hq + d + queries)
    cross(hccs, ctx, rng, [queries, 1, 0, queries - 1], [150, 33, 20, 1], hq, hkv, d, norm, dtype)
    cross(hccs, ctx, rng, [queries], [1203], hq, hkv, d, norm, dtype, fused=True)


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", [(1, 1, 64), (2, 2, 128), (8, 2, 128), (6, 2, 64), (7, 1, 128), (12, 1, 64), (32, 1, 64)])
@pytest.mark.parametrize("k_lens", [(1, 16, 31, 0, 32), (33, 77, 64, 2, 96), (127, 128, 129, 100, 1), (255, 256, 224, 250, 192), (257, 500, 384, 3, 300)])
@pytest.mark.parametrize("norm,dtype", [("div", "i32"), ("clb", "f32"), ("real", "f32"), ("real", "bf16")])
def test_many_queries(hccs, ctx, hq, hkv, d, k_lens, norm, dtype):
    """Lengths around blocks of 32 and 128 keys, tiles of 128 rows cut by the sequences' ends, sequences without queries or keys."""
    rng = np.random.default_rng(hq + d + sum(k_lens))
    cross(hccs, ctx, rng, [129, 40, 0, 17, 300 // hq + 18], k_lens, hq, hkv, d, norm, dtype, fused=hq % 2 == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "i32"])
@pytest.mark.parametrize("d,hq,hkv,length", [(64, 4, 4, 50), (128, 4, 1, 200), (128, 8, 8, 700), (64, 16, 2, 1500)])
def test_shared_states(hccs, ctx, d, hq, hkv, length, dtype):
    rng = np.random.default_rng(length)
    for queries in (1, 30):
        cross(hccs, ctx, rng, [queries, queries, 2, queries], [length, length, 9, length], hq, hkv, d, "div", dtype, share=[0, 0, 2, 0])


@pytest.mark.gpu
@pytest.mark.parametrize("d,hq,hkv", [(64, 3, 3), (128, 2, 1), (64, 12, 2), (128, 9, 1), (64, 20, 1)])
@pytest.mark.parametrize("norm,dtype", [("div", "i32"), ("real", "f32")])
def test_single_queries_of_sequences_with_the_same_states(hccs, ctx, d, hq, hkv, norm, dtype):
    """Runs of hypotheses of one input: longer than a CTA takes together, across its blocks, broken by others, some without a query."""
    rng = np.random.default_rng(d + hq)
    share = [0] * 11 + [11, 12, 12, 12, 15, 12, 17, 17, 11, 11]
    lens = [201] * 11 + [64, 33, 33, 33, 0, 33, 1500, 1500, 64, 64]
    q_lens = [1] * len(lens)
    q_lens[0] = q_lens[4] = q_lens[13] = 0
    cross(hccs, ctx, rng, q_lens, lens, hq, hkv, d, norm, dtype, share=share, theta=_theta(rng, hq, 1500, False))
    cross(hccs, ctx, rng, [0, 0, 1, 0], [70] * 4, hq, hkv, d, norm, dtype, share=[0, 0, 0, 0])


def _some_ranges(rng, q_lens, k_lens):
    out = []
    for nq, n in zip(q_lens, k_lens):
        for i in range(nq):
            kind = rng.integers(0, 6)
            a, b = sorted(int(v) for v in rng.integers(-3, n + 4, 2))
            out.append([(0, 0), (0, n), (a, b), (b, a), (a, a + 1), (0, 1 << 30)][kind])
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 2, 128), (5, 1, 128)])
@pytest.mark.parametrize("norm,dtype", [("div", "i32"), ("real", "f32")])
@pytest.mark.parametrize("q_lens,k_lens", [((1, 1, 1, 1, 0), (40, 1, 300, 0, 9)), ((20, 3, 1), (500, 30, 0)), ((150, 60), (700, 129))])
def test_key_ranges(hccs, ctx, hq, hkv, d, norm, dtype, q_lens, k_lens):
    """Every query its own keys: none, all, one, some in the middle, bounds outside the sequence or in the wrong order."""
    rng = np.random.default_rng(hq + d + sum(k_lens))
    for _ in range(3):
        cross(hccs, ctx, rng, q_lens, k_lens, hq, hkv, d, norm, dtype, ranges=_some_ranges(rng, q_lens, k_lens))


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_key_ranges_of_images(hccs, ctx, d):
    """Texts that see the image they follow: tiles whose rows see one image, two, or none, with whole blocks in the middle."""
    rng = np.random.default_rng(d)
    q_lens, k_lens, per = [500, 200], [2404, 1803], 601
    ranges = []
    for nq, n in zip(q_lens, k_lens):
        at = sorted(int(v) for v in rng.integers(0, nq, n // per))
        for i in range(nq):
            last = sum(a <= i for a in at) - 1
            ranges.append((last * per, last * per + per) if last >= 0 else (0, 0))
    cross(hccs, ctx, rng, q_lens, k_lens, 4, 2, d, "real", "f32", ranges=ranges, wide=True)
    none = [(0, 0)] * 700
    out, _ = cross(hccs, ctx, rng, q_lens, k_lens, 4, 2, d, "real", "f32", ranges=none, wide=True)
    assert (out[:700] == 0).all()


# ------------------------------------------------------------------------------------------- as programs use them
@pytest.mark.gpu
@pytest.mark.parametrize("d,hq,hkv", [(64, 4, 4), (128, 8, 2)])
def test_vision_language_step(hccs, d, hq, hkv):
    """Patches of images with rows and columns through the encoder's attention; its keys and values as states; a prompt and a
    token of the decoder look at them, and write their own keys with three axes into the cache that they attend to."""
    import torch
    from oracle import hccs_oracle as rows
    rng = np.random.default_rng(d)
    B, L, page = 2, 60, 16
    ctx = hccs.Context(0)
    theta = np.array([(100, 1, 60)] * hq, np.int32)
    ctx.hccs_params_upload(theta, 128)
    mult, scale = np.full(hq, 900, np.int32), np.full(hq, 0.03, np.float32)
    steps = [np.full(n, 0.03, np.float32) for n in (hq, hkv, hkv)]
    image = hccs.hccs_rope_axes(d, (d // 4, d // 4), restart=True)
    half = d // 2
    # the encoder: heads first, one kv head per query head
    q, k, v = _tokens(rng, B * L, hq, hq, d, "bf16")
    pos = np.stack([np.tile(np.arange(L) // 10, B), np.tile(np.arange(L) % 10, B)]).astype(np.int32)
    P = torch.from_numpy(pos).cuda()
    q8, k8, v8 = (torch.empty((B, hq, L, d), dtype=torch.int8, device="cuda") for _ in range(3))
    out = torch.empty((B, hq, L, d), dtype=torch.int32, device="cuda")
    ctx.hccs_states_write(q, k, v, q8, k8, v8, P, steps[0], steps[0], steps[0], rope=image)
    ctx.hccs_attention_fused(q8, k8, v8, out, mult, 20)
    freq, axis = list(image.rope.freq)[:half], list(image.axis)[:half]
    turned = [orc.quantise(orc.rotate_axes(t.float().cpu().numpy(), pos, freq, axis, False, 1.0), steps[0]).reshape(B, L, hq, d).transpose(0, 2, 1, 3)
              for t in (q, k)] + [orc.quantise(v.float().cpu().numpy(), steps[0]).reshape(B, L, hq, d).transpose(0, 2, 1, 3)]
    for got, want in zip((q8, k8, v8), turned):
        assert (got.cpu().numpy() == want).all()
    want = rows.attention(*turned, mult, 20, theta)
    assert (out.cpu().numpy() == want).all()
    # the states that the decoder looks at
    _, k, v = _tokens(rng, B * L, hq, hkv, d, "f16")
    k8, v8 = (torch.empty((B * L, hkv, d), dtype=torch.int8, device="cuda") for _ in range(2))
    ctx.hccs_states_write(None, k, v, None, k8, v8, None, None, steps[1], steps[2])
    kk, vv = (orc.quantise(t.float().cpu().numpy(), steps[1]) for t in (k, v))
    k_start, k_len = torch.tensor([0, L], dtype=torch.int32).cuda(), torch.tensor([L, L - 7], dtype=torch.int32).cuda()
    pool_k, pool_v = (torch.zeros((12, hkv, page, d), dtype=torch.int8, device="cuda") for _ in range(2))
    table = torch.tensor([[3, 1, 4], [0, 5, 9]], dtype=torch.int32).cuda()
    text = hccs.hccs_rope_axes(d, (half - 2 * (half // 3), half // 3, half // 3), order=hccs.HCCS_AXES_TURNS)
    done = 0
    for n in (20, 1):                                      # a prompt of two texts, then a token of each
        T = 2 * n
        q, k, v = _tokens(rng, T, hq, hkv, d, "bf16")
        at = np.concatenate([done + np.arange(n)] * 2)
        pos = np.stack([at, at, at]).astype(np.int32)
        slots = torch.tensor([int(table[b, j // page]) * page + j % page for b in range(2) for j in range(done, done + n)]).cuda()
        q8 = torch.empty((T, hq, d), dtype=torch.int8, device="cuda")
        start = torch.tensor([0, n, T], dtype=torch.int32).cuda()
        ctx.hccs_cache_write_axes(q, k, v, q8, pool_k, pool_v, torch.from_numpy(pos).cuda(), slots, *steps, rope=text)
        done += n
        kv_len = torch.full((2,), done, dtype=torch.int32).cuda()
        own, seen = (torch.empty((T, hq, d), dtype=torch.float32, device="cuda") for _ in range(2))
        ctx.hccs_attention_cached(q8, pool_k, pool_v, table, start, kv_len, own, mult, 20, max_q=n, max_kv=done, out_scale=scale, flags=hccs.HCCS_RECIP_REAL)
        ctx.hccs_attention_cross(q8, k8, v8, start, k_start, k_len, seen, mult, 20, max_q=n, max_kv=L, out_scale=scale, flags=hccs.HCCS_RECIP_REAL)
        codes = orc.quantise(orc.rotate_axes(q.float().cpu().numpy(), pos, list(text.rope.freq)[:half], list(text.axis)[:half], False, 1.0), steps[0])
        assert (q8.cpu().numpy() == codes).all()
        compare(own, *orc.attend(codes, pool_k.cpu().numpy(), pool_v.cpu().numpy(), table.cpu().numpy(), [0, n, T], [done, done], theta, mult, 20),
                "real", "f32", scale)
        compare(seen, *orc.cross(codes, kk, vv, [0, n, T], [0, L], [L, L - 7], theta, mult, 20), "real", "f32", scale)
    assert ctx.hccs_device_status() == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("queries,length", [(1, 300), (3, 500), (40, 100), (150, 200), (60, 900)])
def test_cross_captured_replayed_and_on_streams(hccs, ctx, queries, length):
    """Every kernel: the same in a graph replayed on other inputs, and on two streams at once."""
    import torch
    rng = np.random.default_rng(queries)
    hq, hkv, d = 4, 2, 64
    theta = _theta(rng, hq, length, False)
    kv = [rng.integers(-128, 128, (length + 6, 2 * hkv, d), dtype=np.int8) for _ in range(2)]
    outs = [cross(hccs, ctx, rng, [queries], [length], hq, hkv, d, "div", "i32", theta=theta, mult=np.full(hq, 500, np.int32), kv=x)
            for x in kv]
    args = [list(o[1][0]) for o in outs]
    kw = outs[0][1][1]
    want = [o[0].clone() for o in outs]
    for o in outs:
        o[0].fill_(5)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for s, a in zip(streams, args):
            ctx.hccs_attention_cross(*a, **kw, stream=s)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert (o[0][:queries] == w[:queries]).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.hccs_attention_cross(*args[0], **kw)
    for i in range(4):                                     # its inputs take the other call's values and back
        j = i % 2
        for k in range(3):
            args[0][k].copy_(args[1][k] if j else torch.from_numpy(kv[0][:, :hkv] if k == 1 else kv[0][:, hkv:]).cuda() if k else args[0][0])
        if i == 0:
            first = args[0][0].clone()
        args[0][0].copy_(args[1][0] if j else first)
        outs[0][0].fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        assert (outs[0][0][:queries] == want[j][:queries]).all()
    assert ctx.hccs_device_status() == 0


@pytest.mark.gpu
def test_writes_captured_and_replayed(hccs):
    import torch
    rng = np.random.default_rng(1)
    T, hq, hkv, d = 33, 4, 2, 64
    ctx = hccs.Context(0)
    q, k, v = _tokens(rng, T, hq, hkv, d, "bf16")
    steps = [np.full(n, 0.03, np.float32) for n in (hq, hkv, hkv)]
    rope = hccs.hccs_rope_axes(d, (8, 12, 12))
    pos = torch.from_numpy(rng.integers(0, 99, (3, T)).astype(np.int32)).cuda()
    out = [torch.zeros((T, n, d), dtype=torch.int8, device="cuda") for n in (hq, hkv, hkv)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.hccs_states_write(q, k, v, *out, pos, *steps, rope=rope)
    for seed in range(3):
        for t in (q, k, v):
            t.copy_(torch.from_numpy(rng.standard_normal(t.shape).astype(np.float32)).cuda())
        pos.copy_(torch.from_numpy(rng.integers(0, 99, (3, T)).astype(np.int32)).cuda())
        graph.replay()
        torch.cuda.synchronize()
        for t, got, step, turn in zip((q, k, v), out, steps, (True, True, False)):
            x = t.float().cpu().numpy()
            y = orc.rotate_axes(x, pos.cpu().numpy(), list(rope.rope.freq)[:32], list(rope.axis)[:32], False, 1.0) if turn else x
            assert (got.cpu().numpy() == orc.quantise(y, step)).all()
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("queries", [1, 3, 40, 200])
def test_lengths_outside_their_bounds(hccs, ctx, queries):
    """Starts and lengths that leave the states, queries beyond max_q, keys beyond max_kv, starts that leave the tokens: nothing
    outside is read or written, the rest is right, and the status word tells."""
    import torch
    rng = np.random.default_rng(queries)
    hq, hkv, d, S, dev = 4, 2, 64, 90, "cuda"
    theta, mult = _theta(rng, hq, 300, False), np.full(hq, 500, np.int32)
    ctx.hccs_params_upload(theta, 300)
    kv = rng.integers(-128, 128, (S, 2 * hkv, d), dtype=np.int8)
    K, V = (torch.from_numpy(np.ascontiguousarray(x)).to(dev) for x in (kv[:, :hkv], kv[:, hkv:]))
    T = 3 * queries
    q = rng.integers(-128, 128, (T, hq, d), dtype=np.int8)
    for k_start, k_len, starts, max_q, max_kv, real in (
            ([0, 80, 0], [50, 30, 90], [0, queries, 2 * queries, T], queries, 90, ([0, 80, 0], [50, 10, 90])),       # beyond the states
            ([-4, 91, 90], [50, 3, 7], [0, queries, 2 * queries, T], queries, 90, ([0, 0, 0], [0, 0, 0])),
            ([0, 5, 2**31 - 1], [-3, 2**31 - 1, 2**31 - 1], [0, queries, 2 * queries, T], queries, 90, ([0, 5, 0], [0, 85, 0])),
            ([0, 10, 20], [70, 70, 30], [0, queries, 2 * queries, T], queries, 40, ([0, 10, 20], [40, 40, 30])),      # max_kv
            ([0, 10, 20], [70, 60, 30], [0, queries, 2 * queries, T + 50], queries, 90, ([0, 10, 20], [70, 60, 30]))):   # q_start
        out = torch.full((T, hq, d), 77, dtype=torch.int32, device=dev)
        ctx.hccs_attention_cross(torch.from_numpy(q).to(dev), K, V, torch.tensor(starts, dtype=torch.int32, device=dev),
                                 torch.tensor(k_start, dtype=torch.int32, device=dev), torch.tensor(k_len, dtype=torch.int32, device=dev),
                                 out, mult, 20, max_q=max_q, max_kv=max_kv)
        word = ctx.hccs_device_status()
        assert word == (16 if starts[-1] <= T else 0), (word, k_start)
        num, zs, cnt = orc.cross(q, kv[:, :hkv], kv[:, hkv:], [min(s, T) for s in starts], *real, theta, mult, 20)
        compare(out, num, zs, cnt, "div", "i32", None)
    if queries > 1:                                        # queries beyond max_q keep what was there
        out = torch.full((T, hq, d), 77, dtype=torch.int32, device=dev)
        starts = [0, queries, queries + 1, T]
        ctx.hccs_attention_cross(torch.from_numpy(q).to(dev), K, V, torch.tensor(starts, dtype=torch.int32, device=dev),
                                 torch.zeros(3, dtype=torch.int32, device=dev), torch.full((3,), 60, dtype=torch.int32, device=dev), out, mult, 20,
                                 max_q=queries, max_kv=60)
        assert ctx.hccs_device_status() == 16
        num, zs, cnt = orc.cross(q, kv[:, :hkv], kv[:, hkv:], starts, [0] * 3, [60] * 3, theta, mult, 20)
        seen = np.zeros(T, bool)
        for a, b in zip(starts, starts[1:]):
            seen[a:min(b, a + queries)] = True
        got = out.cpu().numpy()
        assert (got[seen] == orc.integer_output(num, zs, cnt, False)[seen]).all() and (got[~seen] == 77).all()


@pytest.mark.gpu
def test_cross_refusals(hccs):
    import torch
    ctx = hccs.Context(0)
    dev = "cuda"
    Q = torch.zeros((6, 4, 64), dtype=torch.int8, device=dev)
    K = torch.zeros((50, 2, 64), dtype=torch.int8, device=dev)
    st, k0, kl = (torch.tensor(x, dtype=torch.int32, device=dev) for x in ([0, 3, 6], [0, 20], [20, 30]))
    O = torch.zeros((6, 4, 64), dtype=torch.float32, device=dev)
    mult, scale = np.full(4, 100, np.int32), np.ones(4, np.float32)

    def call(**kw):
        a = dict(Q=Q, K=K, V=K, st=st, k0=k0, kl=kl, O=O, mult=mult, mq=3, mkv=30, kr=None, scale=scale, flags=0)
        a.update(kw)
        ctx.hccs_attention_cross(a["Q"], a["K"], a["V"], a["st"], a["k0"], a["kl"], a["O"], a["mult"], 20, max_q=a["mq"], max_kv=a["mkv"],
                                 key_range=a["kr"], out_scale=a["scale"], flags=a["flags"])
    with pytest.raises(hccs.HccsError) as ei:
        call()
    assert ei.value.status == hccs.HCCS_ERR_NOT_UPLOADED
    ctx.hccs_params_upload_wide(np.array([(500, 2, 100)] * 4, np.int32), 40)
    for kw, status in ((dict(), hccs.HCCS_ERR_CONSTRAINT), (dict(flags=8, mkv=41), hccs.HCCS_ERR_CONSTRAINT)):
        with pytest.raises(hccs.HccsError) as ei:
            call(**kw)
        assert ei.value.status == status
    call(flags=8)
    ctx.hccs_params_upload(np.array([(300, 1, 10)] * 4, np.int32), 64)
    call()
    wide = torch.zeros((50, 2, 80), dtype=torch.int8, device=dev)
    for kw in (dict(K=K[:, :, :32]), dict(V=K[:40]), dict(K=K.float(), V=K.float()), dict(K=K.cpu()), dict(K=K.transpose(0, 1)[:, :2]),
               dict(K=wide[:, :, :64], V=wide[:, :, :64]), dict(st=st[:2]), dict(st=st.long()), dict(k0=k0[:1]), dict(kl=kl.float()), dict(O=O[:5]),
               dict(Q=Q.cpu()), dict(kr=torch.zeros((6, 2), dtype=torch.int64, device=dev)), dict(kr=torch.zeros((5, 2), dtype=torch.int32, device=dev)),
               dict(mult=mult[:3]), dict(scale=scale[:3])):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(scale=None), dict(O=O.int()), dict(flags=1), dict(mq=-1)):
        with pytest.raises(hccs.HccsError):
            call(**kw)
    # nothing to do, and states that are none
    call(Q=Q[:0], O=O[:0], st=torch.zeros(3, dtype=torch.int32, device=dev))
    call(mq=0)
    O.fill_(3)
    for queries in (3, 1):
        call(K=K[:0], V=K[:0], kl=torch.zeros(2, dtype=torch.int32, device=dev), k0=torch.zeros(2, dtype=torch.int32, device=dev), mq=queries, mkv=0)
        torch.cuda.synchronize()
    assert (O == 0).all() and ctx.hccs_device_status() == 16         # (the second call was short of queries)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("queries,length,hq,hkv,d,ranges", [(1, 70000, 8, 2, 128, False), (5, 4000, 3, 1, 64, False), (300, 250, 16, 2, 128, False), (90, 3001, 12, 3, 64, True)])
def test_large_sums(hccs, ctx, queries, length, hq, hkv, d, ranges):
    """Codes of the largest magnitude, tables of the largest scores: every sum at its limit."""
    rng = np.random.default_rng(length)
    kv = np.where(rng.random((length + 6, 2 * hkv, d)) < 0.5, -128, 127).astype(np.int8)
    kv[:, hkv:] = -128
    q = np.where(rng.random((queries, hq, d)) < 0.5, -128, 127).astype(np.int8)
    theta = np.array([(32767, [1, 127, 0][i % 3], 127) for i in range(hq)], np.int32)
    r = [(int(a), int(a) + 1500) for a in rng.integers(0, length - 1500, queries)] if ranges else None
    cross(hccs, ctx, rng, [queries], [length], hq, hkv, d, "real", "f32", wide=True, theta=theta, q=q, kv=kv, ranges=r,
          mult=np.array([[8191, 40, 0][i % 3] for i in range(hq)], np.int32))
    for shift, m in ((1, 0), (2, 1), (24, 8191), (14, 8190), (14, 1)):
        cross(hccs, ctx, rng, [queries], [length], hq, hkv, d, "real", "f32", wide=True, theta=theta, ranges=r, shift=shift, mult=np.full(hq, m, np.int32))


@pytest.mark.gpu
def test_many_sequences_share_the_device_evenly(hccs, ctx):
    """More sequences than lanes, most of them without queries or keys, tiles of all costs: every row once."""
    rng = np.random.default_rng(8)
    B = 150
    q_lens = [int(n) if rng.random() < 0.5 else 0 for n in rng.integers(1, 60, B)]
    q_lens[7] = 400
    k_lens = [int(n) if rng.random() < 0.9 else 0 for n in rng.integers(1, 257, B)]
    cross(hccs, ctx, rng, q_lens, k_lens, 3, 3, 64, "div", "i32", theta=_theta(rng, 3, 256, False))
    cross(hccs, ctx, rng, [n % 20 for n in q_lens], [min(n, 128) for n in k_lens], 8, 2, 128, "clb", "f16", theta=_theta(rng, 8, 128, False), max_q=20)
    cross(hccs, ctx, rng, [0] * 40 + [1] + [0] * 40, [30] * 81, 20, 1, 64, "div", "i32")


@pytest.mark.gpu
@pytest.mark.parametrize("queries,length", [(1, 200), (40, 60), (40, 200), (60, 500)])
@pytest.mark.parametrize("scale", [1e-30, 3e-38, 1e30])
def test_scales_of_any_size(hccs, ctx, queries, length, scale):
    """Quotients below the normal range of fp32 keep their bits."""
    import torch
    rng = np.random.default_rng(length)
    hq, hkv, d = 4, 2, 64
    out, (args, kw, theta) = cross(hccs, ctx, rng, [queries], [length], hq, hkv, d, "real", "f32", wide=True)
    kw["out_scale"] = np.full(hq, scale, np.float32)
    ctx.hccs_attention_cross(*args, **kw)
    kv = [t.cpu().numpy() for t in args[1:3]]
    num, zs, cnt = orc.cross(args[0].cpu().numpy()[:queries], *kv, [0, queries], [3], [length], theta, args[7], 20)
    want = num / zs[..., None] * np.float64(np.float32(scale))
    got = _values(out[:queries])
    # the product itself may lie below the normal range: half of its last place there is 2^-150
    assert (np.abs(got - want) <= np.abs(want) * 4 * 2.0 ** -24 + 2.0 ** -150).all()


@pytest.mark.gpu
@pytest.mark.parametrize("queries,length", [(1, 900), (3, 300), (50, 120), (90, 220), (70, 700)])
def test_chain_of_calls_without_a_pause(hccs, ctx, queries, length):
    """Every call reads what the one before it writes, or writes what that one reads, and starts while it leaves."""
    import torch
    rng = np.random.default_rng(length)
    hq, hkv, d, n = 4, 2, 64, 6
    theta, mult = _theta(rng, hq, length, False), np.full(hq, 500, np.int32)
    ctx.hccs_params_upload(theta, length)
    steps = [np.full(m, 0.03, np.float32) for m in (hq, hkv, hkv)]
    rope = hccs.hccs_rope_axes(d, (16, 16))
    pos = [torch.from_numpy(rng.integers(0, 50, (2, t)).astype(np.int32)).cuda() for t in (queries, length)]
    q = [torch.from_numpy(rng.standard_normal((queries, hq, d)).astype(np.float32)).cuda() for _ in range(n)]
    kv = [torch.from_numpy(rng.standard_normal((2, length, hkv, d)).astype(np.float32)).cuda() for _ in range(n)]
    q8 = torch.empty((queries, hq, d), dtype=torch.int8, device="cuda")
    k8, v8 = (torch.empty((length, hkv, d), dtype=torch.int8, device="cuda") for _ in range(2))
    start, k0, kl = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, queries], [0], [length]))
    outs = [torch.empty((queries, hq, d), dtype=torch.int32, device="cuda") for _ in range(40)]

    def call(i, out):
        ctx.hccs_states_write(None, kv[i][0], kv[i][1], None, k8, v8, pos[1], None, steps[1], steps[2], rope=rope)
        ctx.hccs_states_write(q[i], None, None, q8, None, None, pos[0], steps[0], None, None, rope=rope)
        ctx.hccs_attention_cross(q8, k8, v8, start, k0, kl, out, mult, 20, max_q=queries, max_kv=length)
    want = []
    for i in range(n):
        out = torch.empty_like(outs[0])
        call(i, out)
        torch.cuda.synchronize()
        want.append(out)
        num, zs, cnt = orc.cross(*(t.cpu().numpy() for t in (q8, k8, v8)), [0, queries], [0], [length], theta, mult, 20)
        compare(out, num, zs, cnt, "div", "i32", None)
    for j, out in enumerate(outs):
        call(j % n, out)
    torch.cuda.synchronize()
    for j, out in enumerate(outs):
        assert torch.equal(out, want[j % n]), j


@pytest.mark.gpu
@pytest.mark.parametrize("queries", [1, 40, 200])
def test_states_beyond_four_gigabytes(hccs, ctx, queries):
    """Keys whose offsets do not fit 32 bits."""
    import torch
    rng = np.random.default_rng(queries)
    hq, hkv, d, S = 128, 128, 128, 150000
    n = 400 if queries == 200 else 200
    states = torch.zeros((S, 2 * hkv, d), dtype=torch.int8, device="cuda")
    tail = rng.integers(-128, 128, (n, 2 * hkv, d), dtype=np.int8)
    states[S - n:] = torch.from_numpy(tail).cuda()
    theta, mult = _theta(rng, hq, n, False), np.full(hq, 400, np.int32)
    ctx.hccs_params_upload(theta, n)
    q = rng.integers(-128, 128, (queries, hq, d), dtype=np.int8)
    out = torch.empty((queries, hq, d), dtype=torch.int32, device="cuda")
    ctx.hccs_attention_cross(torch.from_numpy(q).cuda(), states[:, :hkv], states[:, hkv:], *(torch.tensor(x, dtype=torch.int32, device="cuda") for x in
                             ([0, queries], [S - n], [n])), out, mult, 20, max_q=queries, max_kv=n)
    num, zs, cnt = orc.cross(q, tail[:, :hkv], tail[:, hkv:], [0, queries], [0], [n], theta, mult, 20)
    compare(out, num, zs, cnt, "div", "i32", None)
    assert ctx.hccs_device_status() == 0


I32_MIN, I32_MAX = -2**31, 2**31 - 1


@pytest.mark.gpu
@pytest.mark.parametrize("queries", [1, 3, 40])
@pytest.mark.parametrize("bounds", [(40, I32_MIN), (1, I32_MIN), (I32_MAX, I32_MIN), (I32_MAX, -2), (I32_MIN, I32_MAX), (I32_MAX, I32_MAX),
                                    (I32_MIN, I32_MIN), (5, I32_MAX), (I32_MIN, 3), (I32_MIN, 0)])
def test_key_ranges_with_bounds_of_any_size(hccs, ctx, queries, bounds):
    """Bounds up to the ends of int32: cut to the sequence's keys, whatever lies behind them.  Every sequence has others' states around it."""
    rng = np.random.default_rng(queries)
    k_lens = [100, 0, 90, 1, 300, 64]
    out, _ = cross(hccs, ctx, rng, [queries] * len(k_lens), k_lens, 4, 2, 64, "div", "i32", ranges=[bounds] * (queries * len(k_lens)), gap=0)
    if max(bounds[0], 0) >= bounds[1]:
        assert (out[:queries * len(k_lens)] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("queries,length,ranges", [(1, 60, False), (1, 60, True), (3, 60, False), (40, 60, False), (40, 200, False), (40, 300, False), (40, 60, True)])
def test_starts_of_sequences_without_keys(hccs, ctx, queries, length, ranges):
    """A sequence without keys has none outside the states, wherever it is said to start (padding of a batch, say): nothing is
    reported, and its rows are zeros.  With keys such a start is reported, and none of them is seen."""
    import torch
    rng = np.random.default_rng(queries + length)
    hq, hkv, d, S, dev = 4, 2, 64, length + 20, "cuda"
    theta, mult = _theta(rng, hq, length, False), np.full(hq, 500, np.int32)
    ctx.hccs_params_upload(theta, length)
    K, V = (rng.integers(-128, 128, (S, hkv, d), dtype=np.int8) for _ in range(2))
    k_start, k_len = [-1, 3, S + 1, I32_MIN, I32_MAX, S], [0, length, 0, 0, 0, 0]
    B = len(k_start)
    T = B * queries
    q = rng.integers(-128, 128, (T, hq, d), dtype=np.int8)
    starts = [i * queries for i in range(B + 1)]
    R = torch.tensor([[0, length]] * T, dtype=torch.int32, device=dev) if ranges else None
    for last, word in ((k_len[0], 0), (1, 16)):
        k_len[0] = last
        out = torch.full((T, hq, d), 77, dtype=torch.int32, device=dev)
        ctx.hccs_attention_cross(*(torch.from_numpy(x).to(dev) for x in (q, K, V)), *(torch.tensor(x, dtype=torch.int32, device=dev) for x in
                                 (starts, k_start, k_len)), out, mult, 20, max_q=queries, max_kv=length, key_range=R)
        assert ctx.hccs_device_status() == word
        compare(out, *orc.cross(q, K, V, starts, k_start, [0] + k_len[1:], theta, mult, 20), "div", "i32", None)


@pytest.mark.gpu
def test_outputs_that_are_missing(hccs):
    """What goes with a given input and is None is named, in the writes to dense tensors and to the cache."""
    import torch
    ctx = hccs.Context(0)
    dev = "cuda"
    x = torch.zeros((6, 2, 64), device=dev)
    new = {n: torch.zeros((6, 2, 64), dtype=torch.int8, device=dev) for n in ("q8", "k8", "v8")}
    pools = {n: torch.zeros((1, 2, 16, 64), dtype=torch.int8, device=dev) for n in ("k_pages", "v_pages")}
    slots = torch.arange(6, device=dev)
    steps = [np.full(2, 0.1, np.float32)] * 3
    for gone in ("q8", "k8", "v8"):
        for q, k in ((x, x), (x, None), (None, x)):
            a = dict(new)
            a[gone] = None
            if (q if gone == "q8" else k) is None:             # goes with nothing that is given
                ctx.hccs_states_write(q, k, k, a["q8"], a["k8"], a["v8"], None, *steps)
                continue
            with pytest.raises(ValueError, match=gone):
                ctx.hccs_states_write(q, k, k, a["q8"], a["k8"], a["v8"], None, *steps)
    for gone in ("q8", "k_pages", "v_pages", "slots"):
        for q, k in ((x, x), (x, None), (None, x)):
            for call in (ctx.hccs_cache_write, ctx.hccs_cache_write_axes):
                a = dict(new, **pools, slots=slots)
                a[gone] = None
                if (q if gone == "q8" else k) is None:
                    call(q, k, k, a["q8"], a["k_pages"], a["v_pages"], None, a["slots"], *steps)
                    continue
                with pytest.raises(ValueError, match=gone):
                    call(q, k, k, a["q8"], a["k_pages"], a["v_pages"], None, a["slots"], *steps)
    assert ctx.hccs_device_status() == 0
    ctx.close()


@pytest.mark.gpu
def test_rotations_of_the_other_kind(hccs):
    """Rope and RopeAxes have different layouts: each write takes its own alone."""
    import torch
    ctx = hccs.Context(0)
    dev = "cuda"
    x = torch.zeros((6, 2, 64), device=dev)
    q8, k8, v8 = (torch.zeros((6, 2, 64), dtype=torch.int8, device=dev) for _ in range(3))
    kp, vp = (torch.zeros((1, 2, 16, 64), dtype=torch.int8, device=dev) for _ in range(2))
    slots, steps = torch.arange(6, device=dev), [np.full(2, 0.1, np.float32)] * 3
    one, several = hccs.hccs_rope_frequencies(64), hccs.hccs_rope_axes(64, (16, 16))
    pos1, pos2 = torch.zeros(6, dtype=torch.int32, device=dev), torch.zeros((2, 6), dtype=torch.int32, device=dev)

    def dense(rope, positions):
        ctx.hccs_states_write(x, x, x, q8, k8, v8, positions, *steps, rope=rope)

    def paged(rope, positions):
        ctx.hccs_cache_write_axes(x, x, x, q8, kp, vp, positions, slots, *steps, rope=rope)

    def plain(rope, positions):
        ctx.hccs_cache_write(x, x, x, q8, kp, vp, positions, slots, *steps, rope=rope)
    for call, right, wrong, positions in ((plain, one, several, pos1), (paged, several, one, pos2), (dense, several, one, pos2)):
        call(right, positions)
        call(None, None)
        for bad in (wrong, 64):
            for p in (positions, None):
                with pytest.raises(ValueError, match="rope"):
                    call(bad, p)
    ctx.close()


@pytest.mark.gpu
def test_positions_of_any_strides_in_a_first_call(hccs):
    """The integer types are looked up in the first call that meets one; it takes a transpose as later ones do."""
    import torch
    from paper_2604_02292_b200 import binding
    ctx = hccs.Context(0)
    x = torch.zeros((6, 2, 64), device="cuda")
    q8 = torch.empty((6, 2, 64), dtype=torch.int8, device="cuda")
    rope, step = hccs.hccs_rope_axes(64, (16, 16)), np.full(2, 0.1, np.float32)
    for positions in (torch.zeros((6, 2), dtype=torch.int32, device="cuda").t(), torch.zeros((2, 12), dtype=torch.int32, device="cuda")[:, ::2]):
        binding._I32.clear()
        ctx.hccs_states_write(x, None, None, q8, None, None, positions, step, None, None, rope=rope)
        assert (q8 == 0).all()
    for bad in (torch.zeros((6, 2), device="cuda").t(), torch.zeros((2, 6), dtype=torch.int64, device="cuda")):
        binding._I32.clear()
        with pytest.raises(ValueError):
            ctx.hccs_states_write(x, None, None, q8, None, None, bad, step, None, None, rope=rope)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("queries,length", [(1, 300), (3, 500), (40, 100), (150, 200), (60, 900)])
def test_captured_between_copies_and_other_streams(hccs, ctx, queries, length):
    """Calls captured behind copies and fills, and behind work of another stream that is joined: every input has arrived by then."""
    import torch
    rng = np.random.default_rng(length)
    hq, hkv, d, dev = 4, 2, 64, "cuda"
    theta, mult = _theta(rng, hq, length, False), np.full(hq, 500, np.int32)
    ctx.hccs_params_upload(theta, length)
    steps = [np.full(m, 0.03, np.float32) for m in (hq, hkv, hkv)]
    fresh = [torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(dev) for s in ((queries, hq, d), (length, hkv, d), (length, hkv, d))]
    q, k, v = (torch.zeros_like(t) for t in fresh)
    q8, k8, v8 = (torch.zeros(t.shape, dtype=torch.int8, device=dev) for t in fresh)
    start, k0, kl = (torch.tensor(x, dtype=torch.int32, device=dev) for x in ([0, queries], [0], [length]))
    out = torch.empty((queries, hq, d), dtype=torch.int32, device=dev)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            k.copy_(fresh[1])
            v.copy_(fresh[2])
            ctx.hccs_states_write(None, k, v, None, k8, v8, None, None, steps[1], steps[2])
        q.copy_(fresh[0])
        ctx.hccs_states_write(q, None, None, q8, None, None, None, steps[0], None, None)
        main.wait_stream(side)
        ctx.hccs_attention_cross(q8, k8, v8, start, k0, kl, out, mult, 20, max_q=queries, max_kv=length)
        q8.zero_()
        k8.zero_()
    for _ in range(3):
        for t in fresh:
            t.copy_(torch.from_numpy(rng.standard_normal(t.shape).astype(np.float32)))
        out.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        codes = [orc.quantise(t.cpu().numpy(), s) for t, s in zip(fresh, steps)]
        compare(out, *orc.cross(*codes, [0, queries], [0], [length], theta, mult, 20), "div", "i32", None)
    assert ctx.hccs_device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("queries,hq,ranges", [(1, 16, False), (1, 16, True), (2, 8, False), (4, 2, False), (1, 5, False), (20, 2, False)])
def test_longest_states(hccs, ctx, d, queries, hq, ranges):
    """As many keys as a call may have, in the most rows that the kernel for few rows takes, and in the kernel for many."""
    rng = np.random.default_rng(d + queries)
    n = hccs.HCCS_MAX_CACHE_KEYS
    r = [(n - 5000 * (i + 1), I32_MAX) for i in range(queries)] if ranges else None
    cross(hccs, ctx, rng, [queries], [n], hq, 1, d, "real", "f32", wide=True, ranges=r)


@pytest.mark.gpu
@pytest.mark.parametrize("queries,length", [(1, 100), (4, 100), (40, 100), (40, 200), (40, 400)])
def test_keys_and_values_with_strides_of_their_own(hccs, ctx, queries, length):
    import torch
    rng = np.random.default_rng(length)
    out, (args, kw, _) = cross(hccs, ctx, rng, [queries], [length], 4, 2, 64, "div", "i32", fused=True)
    want = out.clone()
    for K, V in ((args[1].contiguous(), args[2]), (args[1], args[2].contiguous())):
        out.fill_(5)
        ctx.hccs_attention_cross(args[0], K, V, *args[3:], **kw)
        torch.cuda.synchronize()
        assert torch.equal(out[:queries], want[:queries])


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d", [(100, 1, 64), (128, 1, 128), (129, 1, 64), (256, 1, 128), (256, 256, 64), (96, 3, 64)])
@pytest.mark.parametrize("queries,length,ranges", [(1, 700, False), (1, 90, True), (9, 90, False), (9, 250, False), (5, 700, True)])
def test_groups_of_any_size(hccs, ctx, hq, hkv, d, queries, length, ranges):
    """Up to all query heads on one kv head: more than a tile of 128 rows holds, and as many kv heads as there may be."""
    rng = np.random.default_rng(hq)
    q_lens, k_lens = [queries, 1, 0, queries], [length, 3, 5, length // 2]
    cross(hccs, ctx, rng, q_lens, k_lens, hq, hkv, d, "real", "bf16", ranges=_some_ranges(rng, q_lens, k_lens) if ranges else None, wide=True)
