"""Generation over the int8 cache: rotary write, read back, HCCS attention of new tokens.

Codes and integer outputs are compared for equality.  Float outputs: one product of an exact integer with a
rounded factor.  HCCS_RECIP_REAL computes num * (scale / Z): num and Z to fp32 (2^-24 each), the quotient and the
product (2^-24 each), so 4 * 2^-24 relative; the integer modes o * scale: o is below 2^22 * 1 and exact, one
rounding, 2^-24.  A 16-bit output adds its own half step (bf16 2^-8, fp16 2^-11, plus 2^-25 absolute where
fp16 is subnormal).
"""
import ctypes
import math

import numpy as np
import pytest

from oracle import hccs_cache_oracle as orc

TYPES = ("bf16", "f16", "f32")


# ------------------------------------------------------------------------------------------- host only
@pytest.fixture(scope="module")
def binding():
    from paper_2604_02292_b200 import build
    build.build()
    from paper_2604_02292_b200 import binding as b
    return b


def test_rope_frequencies_by_their_formulas(binding):
    b = binding
    for rot, base in ((2, 10000.0), (32, 10000.0), (64, 500000.0), (128, 1e6)):
        plain = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
        r = b.hccs_rope_frequencies(rot, base)
        assert r.rot_dim == rot and r.interleaved == 0 and r.scale == 1.0
        assert np.allclose(list(r.freq)[:rot // 2], plain, rtol=1e-14, atol=0)
        assert not any(list(r.freq)[rot // 2:])
        r = b.hccs_rope_frequencies(rot, base, interleaved=True, kind=b.HCCS_ROPE_LINEAR, factor=4.0)
        assert r.interleaved == 1
        assert np.allclose(list(r.freq)[:rot // 2], [f / 4 for f in plain], rtol=1e-14, atol=0)
        if rot > 2:
            nb = base * 4.0 ** (rot / (rot - 2))
            r = b.hccs_rope_frequencies(rot, base, kind=b.HCCS_ROPE_BASE, factor=4.0)
            assert np.allclose(list(r.freq)[:rot // 2], [nb ** (-2.0 * i / rot) for i in range(rot // 2)], rtol=1e-13, atol=0)
            # the slowest pair turns factor times slower, the fastest as before
            assert math.isclose(r.freq[rot // 2 - 1], plain[-1] / 4, rel_tol=1e-12) and r.freq[0] == 1.0
    r = b.hccs_rope_frequencies(128, 500000.0, kind=b.HCCS_ROPE_WAVELENGTH, factor=8.0, low=1.0, high=4.0, original_len=8192)
    for i in range(64):
        f = 500000.0 ** (-2.0 * i / 128)
        wave = 2 * math.pi / f
        want = f if wave < 8192 / 4 else f / 8 if wave > 8192 else None
        if want is None:
            keep = (8192 / wave - 1.0) / 3.0
            want = (1 - keep) * f / 8 + keep * f
        assert math.isclose(r.freq[i], want, rel_tol=1e-13), i
    r = b.hccs_rope_frequencies(64, 10000.0, kind=b.HCCS_ROPE_DIMENSION, factor=16.0, low=1.0, high=32.0, original_len=4096)
    assert math.isclose(r.scale, 0.1 * math.log(16.0) + 1.0, rel_tol=1e-15)

    def pair_that_turns(n):
        return 64 * math.log(4096 / (n * 2 * math.pi)) / (2 * math.log(10000.0))
    first, last = max(math.floor(pair_that_turns(32.0)), 0), min(math.ceil(pair_that_turns(1.0)), 63)
    for i in range(32):
        f = 10000.0 ** (-2.0 * i / 64)
        keep = 1.0 - min(max((i - first) / (last - first), 0.0), 1.0)
        assert math.isclose(r.freq[i], f * keep + f / 16 * (1 - keep), rel_tol=1e-13), i


def test_rope_refusals(binding):
    b = binding
    bad = [dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=130), dict(rot_dim=-2), dict(base=1.0), dict(base=float("nan")),
           dict(base=float("inf")), dict(kind=5), dict(kind=-1), dict(kind=1, factor=0.5), dict(kind=1, factor=float("inf")),
           dict(kind=2, rot_dim=2, factor=2.0), dict(kind=3, factor=2.0, low=0.0), dict(kind=3, factor=2.0, low=4.0, high=4.0),
           dict(kind=3, factor=2.0, original_len=0.0), dict(kind=4, factor=2.0, high=float("inf"))]
    for kw in bad:
        args = dict(rot_dim=64)
        args.update(kw)
        with pytest.raises(b.HccsError) as ei:
            b.hccs_rope_frequencies(**args)
        assert ei.value.status == b.HCCS_ERR_INVALID_ARG, kw
    assert b.raw().hccs_rope_frequencies(None, 64, 0, 1e4, None) == b.HCCS_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        b.Rope([1.0] * 65)


def _f(*v):
    return np.array(v, dtype=np.float32)


def test_write_and_read_refusals_without_a_gpu(binding):
    """Argument checks that need no context come first; what passes them all ends at the NULL context."""
    b, lib = binding, binding.raw()
    P = 4096                                               # an aligned address that is never read
    two = _f(0.1, 0.1)

    def write(**kw):
        a = dict(q=P, k=P, v=P, type=b.HCCS_F32, qs=64, ks=64, vs=64, pos=P, slots=P, rope=b.Rope([1.0] * 8), q_step=two,
                 k_step=two, v_step=two, q8=P, kp=P, vp=P, T=3, Hq=2, Hkv=2, d=64, pages=4, size=16)
        a.update(kw)
        ptr = {n: (a[n].ctypes.data if a[n] is not None else None) for n in ("q_step", "k_step", "v_step")}
        return lib.hccs_cache_write(None, a["q"], a["k"], a["v"], a["type"], a["qs"], a["ks"], a["vs"], a["pos"], a["slots"],
                                    ctypes.byref(a["rope"]) if a["rope"] else None, ptr["q_step"], ptr["k_step"], ptr["v_step"],
                                    a["q8"], a["kp"], a["vp"], a["T"], a["Hq"], a["Hkv"], a["d"], a["pages"], a["size"], None)
    I, U = b.HCCS_ERR_INVALID_ARG, b.HCCS_ERR_UNSUPPORTED
    assert write() == I                                    # the NULL context
    for kw in (dict(T=-1), dict(type=0), dict(type=9), dict(k=None), dict(v=None), dict(size=24), dict(size=8), dict(size=1 << 17),
               dict(pages=0), dict(Hkv=0), dict(Hkv=257), dict(Hq=0), dict(Hq=257), dict(q_step=None), dict(k_step=_f(0.1, 0.0)),
               dict(v_step=_f(0.1, np.nan)), dict(q_step=_f(np.inf, 0.1)), dict(q_step=_f(-0.1, 0.1)), dict(rope=b.Rope([1.0] * 33)),
               dict(rope=b.Rope([np.inf])), dict(rope=b.Rope([1.0], scale=np.nan)), dict(pos=None), dict(slots=None), dict(q8=None),
               dict(kp=None)):
        assert write(**kw) == I, kw
    for kw in (dict(d=32), dict(d=96), dict(q=P + 8), dict(k=P + 4), dict(v=P + 2), dict(q8=P + 1), dict(kp=P + 8), dict(vp=P + 8),
               dict(qs=65), dict(ks=66), dict(vs=67), dict(type=b.HCCS_BF16, qs=68)):
        assert write(**kw) == U, kw

    def read(**kw):
        a = dict(kp=P, vp=P, table=P, start=P, ks=two, vs=two, ko=P, vo=P, type=b.HCCS_BF16, B=2, mp=3, ml=40, rows=80, Hkv=2, d=64,
                 pages=4, size=16)
        a.update(kw)
        return lib.hccs_cache_read(None, a["kp"], a["vp"], a["table"], a["start"], a["ks"].ctypes.data, a["vs"].ctypes.data, a["ko"],
                                   a["vo"], a["type"], a["B"], a["mp"], a["ml"], a["rows"], a["Hkv"], a["d"], a["pages"], a["size"], None)
    assert read() == I
    for kw in (dict(B=-1), dict(mp=-1), dict(ml=-1), dict(rows=-1), dict(type=0), dict(size=100), dict(pages=0), dict(Hkv=0),
               dict(ks=_f(0.0, 1.0)), dict(kp=None), dict(table=None), dict(start=None)):
        assert read(**kw) == I, kw
    for kw in (dict(d=48), dict(B=65536), dict(kp=P + 8), dict(ko=P + 8), dict(vo=P + 4)):
        assert read(**kw) == U, kw


def test_attention_refusals_without_a_gpu(binding):
    b, lib = binding, binding.raw()
    P = 4096
    I, U = b.HCCS_ERR_INVALID_ARG, b.HCCS_ERR_UNSUPPORTED

    def call(**kw):
        a = dict(Q=P, kp=P, vp=P, table=P, qs=P, kv=P, tree=None, words=0, mult=np.array([100, 100], np.int32), shift=20, scale=_f(1, 1),
                 O=P, type=b.HCCS_F32, T=3, B=2, Hq=2, Hkv=2, d=64, mp=3, pages=4, size=16, mq=2, mkv=40, flags=0)
        a.update(kw)
        return lib.hccs_attention_cached(None, a["Q"], a["kp"], a["vp"], a["table"], a["qs"], a["kv"], a["tree"], a["words"],
                                         a["mult"].ctypes.data if a["mult"] is not None else None, a["shift"],
                                         a["scale"].ctypes.data if a["scale"] is not None else None, a["O"], a["type"], a["T"], a["B"],
                                         a["Hq"], a["Hkv"], a["d"], a["mp"], a["pages"], a["size"], a["mq"], a["mkv"], a["flags"], None)
    assert call() == I                                     # the NULL context
    for kw in (dict(T=-1), dict(B=-1), dict(mp=-1), dict(mq=-1), dict(mkv=-1), dict(flags=1), dict(flags=4), dict(flags=10), dict(type=7),
               dict(scale=None), dict(type=b.HCCS_I32), dict(type=b.HCCS_I32, scale=None, flags=b.HCCS_RECIP_REAL),
               dict(scale=_f(1, np.nan)), dict(mult=None), dict(Hq=3), dict(Hq=0), dict(size=17), dict(shift=0), dict(shift=25),
               dict(mult=np.array([-1, 0], np.int32)), dict(mult=np.array([1 << 13, 0], np.int32)), dict(tree=P, words=0),
               dict(tree=P, words=1, mq=33), dict(Q=None), dict(table=None), dict(qs=None), dict(kv=None), dict(O=None)):
        assert call(**kw) == I, kw
    for kw in (dict(d=80), dict(B=65536), dict(mkv=131073), dict(Hq=258), dict(shift=5), dict(Q=P + 1), dict(kp=P + 8), dict(vp=P + 8),
               dict(O=P + 4), dict(mq=(1 << 30) + 1)):
        assert call(**kw) == U, kw
    assert lib.hccs_params_upload_wide(None, None, 1, 1, None, None) == I


def test_oracle_of_the_cache_agrees_with_the_row_oracle(oracle):
    """One query that sees every key: the attention oracle's scores are those of the row oracle's int16 path."""
    rng = np.random.default_rng(5)
    n, d, theta = 96, 64, (300, 3, 60)
    q = rng.integers(-64, 64, (1, 1, d), dtype=np.int8)
    k, v = (rng.integers(-64, 64, (6, 1, 16, d), dtype=np.int8) for _ in range(2))
    table = np.array([[3, 1, 5, 0, 2, 4]])
    num, zs, cnt = orc.attend(q, k, v, table, [0, 1], [n], [theta], [2000], 20)
    ks, vs = orc.sequence(k, table[0], n)[:, 0].astype(np.int64), orc.sequence(v, table[0], n)[:, 0].astype(np.int64)
    x = np.clip((ks @ q[0, 0].astype(np.int64) * 2000 + (1 << 19)) >> 20, -128, 127).astype(np.int8)
    for clb, mode in ((False, oracle.MODE_U16), (True, oracle.MODE_U16 | oracle.MODE_CLB)):
        p = oracle.forward(x.reshape(1, 1, 1, n), np.array([theta], np.int32), mode).reshape(n).astype(np.int64)
        assert (orc.integer_output(num, zs, cnt, clb)[0, 0] == p @ vs).all()


# ------------------------------------------------------------------------------------------- helpers
def _torch_type(name):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i32": torch.int32}[name]


def _values(t):
    import torch
    return t.detach().to("cpu", torch.float32).numpy().astype(np.float64)


class Cache:
    """Pools of random codes with shuffled pages, larger than the sequences need."""

    def __init__(self, rng, lens, hkv, d, page, extra=2):
        per = max(-(-max(max(lens), 1) // page), 1)
        pages = per * len(lens) + extra
        self.k, self.v = (rng.integers(-128, 128, (pages, hkv, page, d), dtype=np.int8) for _ in range(2))
        self.table = rng.permutation(pages)[:per * len(lens)].reshape(len(lens), per).astype(np.int32)


def _theta(rng, hq, n, wide):
    out = []
    for _ in range(hq):
        if wide:
            D, S = int(rng.integers(1, 128)), int(rng.integers(0, 128))
            out.append((max(1, S * D + int(rng.integers(0, 200))), S, D))
        else:
            f, top = -(-256 // n), 32767 // n
            D = int(rng.integers(1, max(1, min(127, top - f)) + 1))
            S = int(rng.integers(0, min(127, (top - f) // D) + 1))
            out.append((int(rng.integers(S * D + f, top + 1)), S, D))
    return np.array(out, dtype=np.int32)


def _tree(rng, lens, words):
    rows = []
    for n in lens:
        seen = []
        for i in range(n):
            p = int(rng.integers(-1, i)) if i else -1
            seen.append((seen[p] if p >= 0 else 0) | (1 << i))
        rows += [[(s >> (32 * w)) & 0xFFFFFFFF for w in range(words)] for s in seen]
    return np.array(rows, dtype=np.uint64).astype(np.uint32).view(np.int32).reshape(-1, words)


def attend(pkg, ctx, rng, q_lens, kv_lens, hq, hkv, d, page, norm="real", dtype="f32", tree=None, wide=False, shift=20, mult=None,
           spread=24.0, n_design=None, q=None, theta=None, cache=None, check=True, stream=None):
    """One call and its comparison with the oracle; returns (output tensor, cache, arguments)."""
    import torch
    cache = cache or Cache(rng, kv_lens, hkv, d, page)
    T = sum(q_lens)
    start = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
    q = rng.integers(-128, 128, (T, hq, d), dtype=np.int8) if q is None else q
    n = n_design or max(max(kv_lens), 1)
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
    mask = None
    if tree is not None:
        mask = torch.zeros((T + 2, tree.shape[1]), dtype=torch.int32, device=dev)
        mask[:T] = torch.from_numpy(tree).to(dev)
    args = (Q, torch.from_numpy(cache.k).to(dev), torch.from_numpy(cache.v).to(dev), torch.from_numpy(cache.table).to(dev),
            torch.from_numpy(start).to(dev), torch.tensor(kv_lens, dtype=torch.int32, device=dev), out, mult, shift)
    flags = {"real": pkg.HCCS_RECIP_REAL, "div": 0, "clb": pkg.HCCS_RECIP_CLB}[norm]
    kw = dict(max_q=max(max(q_lens), 1), max_kv=max(max(kv_lens), 1), tree_mask=mask, out_scale=None if dtype == "i32" else scale, flags=flags)
    ctx.hccs_attention_cached(*args, **kw)
    torch.cuda.synchronize()
    assert (_values(out[T:]) == 77).all(), "rows behind the last sequence were written"
    if check:
        num, zs, cnt = orc.attend(q, cache.k, cache.v, cache.table, start, kv_lens, theta, mult, shift, tree)
        compare(out[:T], num, zs, cnt, norm, dtype, scale)
        assert ctx.hccs_device_status() == 0
    return out, cache, (args, kw, theta)


def compare(out, num, zs, cnt, norm, dtype, scale):
    import torch
    if norm == "real":
        want = num / np.maximum(zs, 1)[..., None] * scale.astype(np.float64)[None, :, None]
        rel = 4 * 2.0 ** -24
    else:
        ints = orc.integer_output(num, zs, cnt, norm == "clb")
        if dtype == "i32":
            got = out.cpu().numpy()
            assert (got == ints).all(), f"{(got != ints).sum()} of {got.size} differ, first at {tuple(np.argwhere(got != ints)[0])}"
            return
        want = ints * scale.astype(np.float64)[None, :, None]
        rel = 2.0 ** -24
    step, floor = {"f32": (0.0, 0.0), "bf16": (2.0 ** -8, 0.0), "f16": (2.0 ** -11, 2.0 ** -25)}[dtype]
    got = _values(out)
    off = np.abs(got - want)
    tol = np.abs(want) * (rel + step + rel * step) + floor
    if dtype == "f16":                                    # beyond the type's range the output is infinite
        big = np.abs(want) >= 65520 * (1 - rel)
        assert np.isinf(got[big]).all() if big.any() else True
        off, tol = off[~big], tol[~big]
    assert (off <= tol).all(), f"{(off > tol).sum()} of {off.size} off, worst {np.max(off - tol)}"
    assert (got[cnt == 0] == 0).all()


# ------------------------------------------------------------------------------------------- write and read
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hq,hkv,d,page,rot,interleaved,T", [
    (4, 2, 64, 16, 64, False, 1), (4, 2, 128, 32, 128, False, 37), (3, 3, 64, 16, 32, True, 50), (5, 1, 128, 64, 64, True, 33),
    (2, 2, 64, 16, 0, False, 20), (8, 2, 128, 16, 34, False, 19), (6, 3, 64, 128, 6, True, 23), (2, 1, 64, 16, 20, False, 5),
    (7, 7, 128, 16, 96, False, 40), (16, 4, 64, 16, 2, False, 300)])
def test_write(hccs, dtype, hq, hkv, d, page, rot, interleaved, T):
    import torch
    rng = np.random.default_rng(hq * 1000 + d + T)
    pages = -(-T // page) + 2
    x = torch.from_numpy(rng.standard_normal((T, (hq + 2 * hkv) * d + 16)).astype(np.float32)).to("cuda", _torch_type(dtype))
    q, k, v = (x[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in ((0, hq), (hq, hq + hkv), (hq + hkv, hq + 2 * hkv)))
    pos = rng.integers(0, 131072, T).astype(np.int32)
    pos[0] = 0
    slots = rng.permutation(pages * page)[:T].astype(np.int64)
    if T > 3:
        slots[2] = -1
    steps = [rng.uniform(0.005, 0.05, n).astype(np.float32) for n in (hq, hkv, hkv)]
    steps[0][0] = 0.03125                                  # powers of two: exact ties
    steps[2][0] = 2.0 ** -6
    freq, scale = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)], 1.0 if T % 2 else 1.23
    kp, vp = (rng.integers(-128, 128, (pages, hkv, page, d), dtype=np.int8) for _ in range(2))
    ctx = hccs.Context(0)
    q8 = torch.full((T, hq, d), 99, dtype=torch.int8, device="cuda")
    dk, dv = torch.from_numpy(kp).cuda(), torch.from_numpy(vp).cuda()
    ctx.hccs_cache_write(q, k, v, q8, dk, dv, torch.from_numpy(pos).cuda(), torch.from_numpy(slots).cuda(), *steps,
                         rope=hccs.Rope(freq, interleaved=interleaved, scale=scale) if rot else None)
    assert ctx.hccs_device_status() == 0
    xq, xk, xv = (t.float().cpu().numpy() for t in (q, k, v))
    want_q = orc.quantise(orc.rotate(xq, pos, freq, interleaved, scale), steps[0])
    want_k = orc.write(kp, orc.quantise(orc.rotate(xk, pos, freq, interleaved, scale), steps[1]), slots)
    want_v = orc.write(vp, orc.quantise(xv, steps[2]), slots)
    for name, got, want in (("q", q8, want_q), ("k", dk, want_k), ("v", dv, want_v)):
        assert (got.cpu().numpy() == want).all(), name
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_write_of_infinities_nan_and_the_largest_values(hccs, dtype):
    import torch
    d, T = 64, 6
    big = {"bf16": 3.3895313892515355e38, "f16": 65504.0, "f32": 3.4028234663852886e38}[dtype]
    x = np.zeros((T, 1, d), np.float32)
    x[0, 0, ::3] = np.inf
    x[1, 0, 5] = np.nan
    x[2, 0] = big
    x[3, 0] = -big
    x[4, 0, ::2] = -np.inf
    x[5, 0, :] = np.linspace(-9, 9, d)
    t = torch.from_numpy(x).to("cuda", _torch_type(dtype))
    pos = torch.tensor([0, 1, 0, 70000, 3, -5], dtype=torch.int32, device="cuda")
    freq = [10000.0 ** (-2.0 * i / d) for i in range(d // 2)]
    kp, vp = (torch.zeros((1, 1, 16, d), dtype=torch.int8, device="cuda") for _ in range(2))
    q8 = torch.zeros((T, 1, d), dtype=torch.int8, device="cuda")
    ctx = hccs.Context(0)
    slots = torch.arange(T, device="cuda")
    ctx.hccs_cache_write(t, t, t, q8, kp, vp, pos, slots, [0.05], [0.07], [0.07], rope=hccs.Rope(freq))
    xs = t.float().cpu().numpy()
    want = orc.rotate(xs, pos.cpu().numpy(), freq, False, 1.0)
    assert (q8.cpu().numpy() == orc.quantise(want, [0.05])).all()
    assert (kp[0, 0, :T].cpu().numpy() == orc.quantise(want, [0.07])[:, 0]).all()
    assert (vp[0, 0, :T].cpu().numpy() == orc.quantise(xs.astype(np.longdouble), [0.07])[:, 0]).all()
    assert not kp[0, 0, T:].any() and not vp[0, 0, T:].any()
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("step", [0.03, 0.03125, 1.0, 0.3333333, 7e-3, 1e-6, 1e30, 2.0 ** -100, 2.0 ** 100, 3e30, 1.1754944e-38, 2.0 ** -140])
def test_write_at_the_borders(hccs, dtype, step):
    """Values on, just below and just above every border k + 1/2, and all 16-bit patterns of the type's range."""
    import torch
    s = np.float32(step)
    k = np.arange(-130, 130)
    v = ((k + 0.5) * np.float64(s)).astype(np.float32)
    vals = np.concatenate([v, np.nextafter(v, np.float32(-np.inf)), np.nextafter(v, np.float32(np.inf)), (k * np.float64(s)).astype(np.float32)])
    bits = torch.from_numpy(np.arange(0, 65536, 1, dtype=np.uint16).view(np.int16))
    some = {"bf16": bits.view(torch.bfloat16), "f16": bits.view(torch.float16), "f32": bits.view(torch.bfloat16).float()}[dtype]
    x = torch.cat([torch.from_numpy(vals).to(_torch_type(dtype)), some])
    x = torch.cat([x, x[:-x.numel() % 64]]) if x.numel() % 64 else x
    x = x.view(-1, 1, 64).cuda()
    T = x.shape[0]
    pages = -(-T // 16)
    kp, vp = (torch.zeros((pages, 1, 16, 64), dtype=torch.int8, device="cuda") for _ in range(2))
    q8 = torch.zeros((T, 1, 64), dtype=torch.int8, device="cuda")
    ctx = hccs.Context(0)
    args = (x, x, x, q8, kp, vp, torch.zeros(T, dtype=torch.int32, device="cuda"), torch.arange(T, device="cuda"), [s], [s], [s])
    if step < 2.0 ** -100 or step > 2.0 ** 100:            # a reciprocal that fp32 cannot hold: refused
        with pytest.raises(hccs.HccsError) as ei:
            ctx.hccs_cache_write(*args)
        assert ei.value.status == hccs.HCCS_ERR_INVALID_ARG
        return
    ctx.hccs_cache_write(*args, rope=hccs.Rope([1.0] * 16))                                    # position 0: turned by nothing
    xs = x.float().cpu().numpy()
    with np.errstate(invalid="ignore"):                    # (signalling NaNs among the patterns)
        want = orc.quantise(xs.astype(np.longdouble), [s])
    assert (vp.cpu().numpy().reshape(-1, 64)[:T] == want[:, 0]).all()
    finite = np.isfinite(xs).all(axis=(1, 2))              # an infinity times a sine of zero is a NaN
    assert (q8.cpu().numpy()[finite] == want[finite]).all() and (kp.cpu().numpy().reshape(-1, 64)[:T][finite] == want[finite][:, 0]).all()
    ctx.close()


@pytest.mark.gpu
def test_write_parts_and_bad_slots(hccs):
    import torch
    ctx = hccs.Context(0)
    x = torch.randn(4, 2, 64, device="cuda")
    pool = [torch.full((2, 2, 16, 64), 11, dtype=torch.int8, device="cuda") for _ in range(2)]
    q8 = torch.full((4, 2, 64), 11, dtype=torch.int8, device="cuda")
    step = np.array([0.02, 0.03], np.float32)
    ctx.hccs_cache_write(x, None, None, q8, None, None, None, None, step, None, None)          # queries alone
    assert (q8.cpu().numpy() == orc.quantise(x.cpu().numpy().astype(np.longdouble), step)).all()
    slots = torch.tensor([3, 32, -7, 1 << 40], device="cuda")                                  # the second and the fourth lie beyond the pools
    ctx.hccs_cache_write(None, x, x, None, *pool, None, slots, None, step, step)               # keys and values alone
    codes = orc.quantise(x.cpu().numpy().astype(np.longdouble), step)
    for p in pool:
        assert (p.cpu().numpy() == orc.write(np.full((2, 2, 16, 64), 11, np.int8), codes, [3, -1, -1, -1])).all()
    assert ctx.hccs_device_status() == 4 and ctx.hccs_device_status() == 0
    ctx.hccs_cache_write(x[:0], x[:0], x[:0], q8[:0], *pool, None, slots[:0], step, step, step)   # no token
    with pytest.raises(ValueError):
        ctx.hccs_cache_write(x, x, None, q8, *pool, None, slots, step, step, step)
    with pytest.raises(ValueError):
        ctx.hccs_cache_write(x.cpu(), x, x, q8, *pool, None, slots, step, step, step)
    with pytest.raises(ValueError):
        ctx.hccs_cache_write(x.transpose(1, 2).contiguous().transpose(1, 2), x, x, q8, *pool, None, slots, step, step, step)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("lens,hkv,d,page", [([1], 1, 64, 16), ([0, 33, 16, 0, 1], 3, 64, 16), ([130, 257], 8, 128, 64), ([1000], 2, 128, 16),
                                             ([5, 511, 90], 12, 64, 512)])
def test_read(hccs, dtype, lens, hkv, d, page):
    import torch
    rng = np.random.default_rng(len(lens) * 10 + hkv)
    c = Cache(rng, lens, hkv, d, page)
    start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    total = int(start[-1])
    out = [torch.full((total + 3, hkv, d), -5, dtype=_torch_type(dtype), device="cuda") for _ in range(2)]
    steps = [rng.uniform(0.001, 0.1, hkv).astype(np.float32) for _ in range(2)]
    ctx = hccs.Context(0)
    pools = (torch.from_numpy(c.k).cuda(), torch.from_numpy(c.v).cuda())
    args = (torch.from_numpy(c.table).cuda(), torch.from_numpy(start).cuda())
    ctx.hccs_cache_read(*pools, *args, *out, *steps, max(lens))
    assert ctx.hccs_device_status() == 0
    for got, pool, step in zip(out, (c.k, c.v), steps):
        seqs = np.concatenate([orc.sequence(pool, c.table[b], n) for b, n in enumerate(lens)])
        want = torch.from_numpy(seqs.astype(np.float32) * step[None, :, None]).to(_torch_type(dtype))     # fp32 product, rounded to the type
        assert torch.equal(got[:total].cpu(), want)
        assert (_values(got[total:]) == -5).all()
    one = torch.full_like(out[0], -5)                      # one of the two alone
    ctx.hccs_cache_read(*pools, *args, None, one, *steps, max(lens))
    assert torch.equal(one, out[1])
    ctx.close()


@pytest.mark.gpu
def test_read_reports_what_is_out_of_range(hccs):
    import torch
    ctx = hccs.Context(0)
    pool = torch.randint(-128, 128, (3, 1, 16, 64), device="cuda").to(torch.int8)
    table = torch.tensor([[0, 7], [-1, 2]], dtype=torch.int32, device="cuda")
    start = torch.tensor([0, 20, 52], dtype=torch.int32, device="cuda")
    out = [torch.full((52, 1, 64), -5.0, device="cuda") for _ in range(2)]
    ctx.hccs_cache_read(pool, pool, table, start, *out, [1.0], [1.0], 32)
    for o in out:
        assert torch.equal(o[:16, 0], pool[0, 0].float()) and not o[16:36].any() and torch.equal(o[36:52, 0], pool[2, 0].float())
    assert ctx.hccs_device_status() == 8
    short = [torch.full((30, 1, 64), -5.0, device="cuda") for _ in range(2)]                # cut at the outputs' end and at max_len
    ctx.hccs_cache_read(pool, pool, table.clamp(0, 2), start, *short, [1.0], [1.0], 12)
    for o in short:
        assert torch.equal(o[:12, 0], pool[0, 0, :12].float()) and (o[12:20] == -5).all() and torch.equal(o[20:30, 0], pool[0, 0, :10].float())
    assert ctx.hccs_device_status() == 16
    ctx.close()


# ------------------------------------------------------------------------------------------- attention
@pytest.mark.gpu
@pytest.mark.parametrize("norm,dtype", [("div", "i32"), ("clb", "i32"), ("real", "f32"), ("real", "bf16"), ("real", "f16"), ("div", "f32"), ("clb", "bf16")])
@pytest.mark.parametrize("hq,hkv,d,page", [(4, 4, 64, 16), (8, 2, 128, 64), (14, 2, 64, 32)])
def test_single_tokens(hccs, norm, dtype, hq, hkv, d, page):
    ctx = hccs.Context(0)
    rng = np.random.default_rng(1)
    kv = [1, 2, 15, 16, 17, 31, 33, 100, 129, 500, 513]
    attend(hccs, ctx, rng, [1] * len(kv), kv, hq, hkv, d, page, norm, dtype)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv", [(1, 1), (2, 1), (3, 1), (5, 1), (7, 1), (8, 1), (9, 1), (12, 1), (15, 1), (16, 1), (17, 1), (24, 1), (33, 1), (64, 2), (256, 4), (130, 1)])
def test_head_groups(hccs, hq, hkv):
    ctx = hccs.Context(0)
    rng = np.random.default_rng(hq)
    attend(hccs, ctx, rng, [1, 1], [200, 77], hq, hkv, 64, 16, "div", "i32")
    attend(hccs, ctx, rng, [3, 1], [90, 130], hq, hkv, 128, 32, "real", "f32")
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("wide", [False, True])
def test_long_caches_of_single_tokens(hccs, d, wide):
    ctx = hccs.Context(0)
    rng = np.random.default_rng(3)
    attend(hccs, ctx, rng, [1, 1, 1], [8191, 2000, 4097] if wide else [4000, 3999, 17], 8, 2, d, 64, "real", "f32", wide=wide)
    attend(hccs, ctx, rng, [1], [20011 if wide else 1025], 4, 1, d, 16, "real", "bf16", wide=wide)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("q_lens,kv_lens", [([5], [5]), ([1, 4, 0, 9], [300, 4, 20, 64]), ([40, 130], [40, 700]), ([300], [300]), ([17, 64, 128], [500, 64, 129]),
                                            ([129, 1, 2], [1000, 1000, 2])])
@pytest.mark.parametrize("hq,hkv,d,page,norm,dtype", [(4, 2, 64, 16, "div", "i32"), (6, 2, 128, 64, "real", "f32"), (2, 2, 128, 16, "clb", "i32"), (3, 1, 64, 256, "real", "bf16")])
def test_causal_queries(hccs, q_lens, kv_lens, hq, hkv, d, page, norm, dtype):
    ctx = hccs.Context(0)
    rng = np.random.default_rng(sum(q_lens))
    attend(hccs, ctx, rng, q_lens, kv_lens, hq, hkv, d, page, norm, dtype)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("q_lens,kv_lens", [([1], [40]), ([7, 13, 1], [7, 700, 30]), ([32, 33, 64], [200, 129, 640]), ([70, 5], [1024, 133]), ([200], [333])])
@pytest.mark.parametrize("hq,hkv,d,page,norm,dtype", [(4, 1, 64, 16, "clb", "i32"), (8, 2, 128, 64, "real", "f32"), (3, 3, 128, 128, "div", "i32")])
def test_trees(hccs, q_lens, kv_lens, hq, hkv, d, page, norm, dtype):
    ctx = hccs.Context(0)
    rng = np.random.default_rng(sum(q_lens) + 1)
    attend(hccs, ctx, rng, q_lens, kv_lens, hq, hkv, d, page, norm, dtype, tree=_tree(rng, q_lens, -(-max(q_lens) // 32)))
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("B,q_len,kv,hq,hkv,d,page", [(8, 8, 8000, 32, 8, 128, 64), (8, 8, 7900, 32, 8, 64, 16), (3, 100, 6001, 8, 4, 128, 32), (40, 3, 2305, 16, 4, 64, 128),
                                                      (2, 700, 5000, 12, 4, 128, 64), (1, 5, 60000, 6, 1, 128, 16), (1, 1000, 1000, 30, 10, 64, 32), (20, 40, 4100, 8, 8, 128, 256)])
def test_many_queries_agree_with_single_tokens(hccs, B, q_len, kv, hq, hkv, d, page):
    """At sizes beyond the oracle: a causal query is a single token of a sequence that ends with it, and sums are exact,
    so both kernels give the same bits.  Repeated, since what could go wrong here are races."""
    import torch
    rng = np.random.default_rng(kv)
    ctx = hccs.Context(0)
    ctx.hccs_params_upload_wide(_theta(rng, hq, kv, True), kv)
    g = torch.Generator(device="cuda").manual_seed(kv)
    per = -(-kv // page)
    kp, vp = (torch.randint(-128, 128, (B * per, hkv, page, d), device="cuda", generator=g).to(torch.int8) for _ in range(2))
    table = torch.randperm(B * per, device="cuda", generator=g).to(torch.int32).reshape(B, per)
    Q = torch.randint(-128, 128, (B * q_len, hq, d), device="cuda", generator=g).to(torch.int8)
    mult, scale = np.full(hq, int(20 / (74.0 ** 2 * math.sqrt(d)) * (1 << 20)), np.int32), np.full(hq, 0.03, np.float32)
    lens = torch.randint(q_len + (kv - q_len) // 2, kv + 1, (B,), device="cuda", generator=g).to(torch.int32)
    lens[0] = kv
    kw = dict(out_scale=scale, flags=hccs.HCCS_RECIP_REAL, max_kv=kv)
    want = torch.empty((B * q_len, hq, d), device="cuda")
    single = lens.repeat_interleave(q_len) - q_len + 1 + torch.arange(q_len, device="cuda", dtype=torch.int32).repeat(B)
    ctx.hccs_attention_cached(Q, kp, vp, table.repeat_interleave(q_len, 0).contiguous(), torch.arange(B * q_len + 1, dtype=torch.int32, device="cuda"),
                              single.to(torch.int32), want, mult, 20, max_q=1, **kw)
    start = torch.arange(0, B * q_len + 1, q_len, dtype=torch.int32, device="cuda")
    for _ in range(8):
        got = torch.full_like(want, 7.0)
        ctx.hccs_attention_cached(Q, kp, vp, table, start, lens, got, mult, 20, max_q=q_len, **kw)
        assert ctx.hccs_device_status() == 0
        assert torch.equal(got, want), f"{(got != want).sum().item()} of {got.numel()} differ"
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_rows_that_see_nothing(hccs, d):
    """Tree rows without a bit and without a prefix, queries in front of the first key, sequences without keys."""
    ctx = hccs.Context(0)
    rng = np.random.default_rng(9)
    tree = _tree(rng, [6, 1, 1], 1)
    tree[2] = 0
    tree[6:] = 0
    for norm, dtype in (("div", "i32"), ("real", "f32")):
        attend(hccs, ctx, rng, [6, 1, 1], [6, 1, 40], 4, 2, d, 16, norm, dtype, tree=tree)
        attend(hccs, ctx, rng, [6, 3], [2, 0], 4, 2, d, 16, norm, dtype)
        attend(hccs, ctx, rng, [1, 1, 1], [0, 5, 0], 4, 2, d, 16, norm, dtype)
        tree1 = np.array([[0], [1], [0]], np.int32)
        attend(hccs, ctx, rng, [1, 1, 1], [1, 1, 9], 4, 2, d, 16, norm, dtype, tree=tree1)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("shift,mult", [(20, 0), (1, 0), (14, 8191), (24, 8191), (20, 8191), (20, 1), (4, 7), (10, 511)])
@pytest.mark.parametrize("q_len", [1, 9])
def test_requantisation_range(hccs, shift, mult, q_len):
    """Logits that all saturate, that all are zero, and the largest steps."""
    ctx = hccs.Context(0)
    rng = np.random.default_rng(shift + mult)
    for d in (64, 128):
        attend(hccs, ctx, rng, [q_len, q_len], [150, 60], 4, 2, d, 16, "div", "i32", shift=shift, mult=np.array([mult] * 4, np.int32))
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("q_len", [1, 4])
def test_extreme_codes_and_tables(hccs, q_len):
    """All codes at -128 (the largest accumulators), and tables at the ends of both bands."""
    ctx = hccs.Context(0)
    rng = np.random.default_rng(2)
    c = Cache(rng, [300], 2, 128, 16)
    c.k[:], c.v[:] = -128, -128
    q = np.full((q_len, 4, 128), -128, np.int8)
    for theta, wide, norm in (([(1, 0, 127)] * 4, True, "real"), ([(32767, 127, 127), (127 * 127, 127, 127), (1, 1, 1), (32767, 0, 1)], True, "real"),
                              ([(109, 0, 1), (1, 0, 1), (109, 1, 108), (2, 1, 1)], False, "div")):
        attend(hccs, ctx, rng, [q_len], [300], 4, 2, 128, 16, norm, "i32" if norm == "div" else "f32", wide=wide, theta=np.array(theta, np.int32),
               q=q, cache=c, mult=np.array([8191, 100, 1, 0], np.int32))
    ctx.close()


@pytest.mark.gpu
def test_table_kinds_and_refusals(hccs):
    import torch
    ctx = hccs.Context(0)
    rng = np.random.default_rng(4)
    out, c, (args, kw, theta) = attend(hccs, ctx, rng, [1, 1], [30, 20], 4, 2, 64, 16, "real", "f32", wide=True, n_design=64)
    x = torch.zeros((1, 4, 8, 64), dtype=torch.int8, device="cuda")
    p = torch.zeros((1, 4, 8, 64), dtype=torch.uint8, device="cuda")
    o = torch.zeros((1, 4, 8, 64), dtype=torch.int32, device="cuda")
    for call in (lambda: ctx.hccs_forward(x, p), lambda: ctx.hccs_attention_fused(x, x, x, o, [100] * 4, 20),
                 lambda: ctx.hccs_attention_cached(*args, **{**kw, "flags": 0}), lambda: ctx.hccs_attention_cached(*args, **{**kw, "max_kv": 65})):
        with pytest.raises(hccs.HccsError) as ei:
            call()
        assert ei.value.status == hccs.HCCS_ERR_CONSTRAINT
    with pytest.raises(hccs.HccsError) as ei:
        ctx.hccs_params_upload_wide([(10, 1, 5), (10, 2, 6)], 64)
    assert ei.value.status == hccs.HCCS_ERR_CONSTRAINT and "head 1" in str(ei.value)
    for n in (0, 131073):
        with pytest.raises(hccs.HccsError) as ei:
            ctx.hccs_params_upload_wide([(10, 1, 5)], n)
        assert ei.value.status == hccs.HCCS_ERR_INVALID_ARG
    ctx.hccs_params_upload([(300, 3, 85)] * 4, 64)         # an ordinary table again: the other calls run
    ctx.hccs_forward(x, p)
    fresh = hccs.Context(0)
    with pytest.raises(hccs.HccsError) as ei:
        fresh.hccs_attention_cached(*args, **kw)
    assert ei.value.status == hccs.HCCS_ERR_NOT_UPLOADED
    fresh.hccs_params_upload([(300, 3, 85)] * 2, 64)
    with pytest.raises(hccs.HccsError) as ei:
        fresh.hccs_attention_cached(*args, **kw)           # another number of heads
    assert ei.value.status == hccs.HCCS_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        ctx.hccs_attention_cached(args[0].cpu(), *args[1:], **kw)
    fresh.close()
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("q_len", [1, 5])
def test_bad_pages_and_lengths_are_reported(hccs, q_len):
    """A page outside the pools hides its keys; lengths beyond their bounds are cut."""
    import torch
    rng = np.random.default_rng(8)
    ctx = hccs.Context(0)
    out, c, (args, kw, theta) = attend(hccs, ctx, rng, [q_len], [64], 4, 2, 64, 16, "div", "i32")
    pages = c.k.shape[0]
    for bad in (pages, -1, 2 ** 31 - 1):
        table = c.table.copy()
        table[0, 1] = bad
        a = list(args)
        a[3] = torch.from_numpy(table).cuda()
        ctx.hccs_attention_cached(*a, **kw)
        assert ctx.hccs_device_status() == 8
        # the same as the other three pages alone, with the new tokens at the end
        short = c.table[:, [0, 2, 3]].copy()
        num, zs, cnt = orc.attend(args[0][:q_len].cpu().numpy(), c.k, c.v, short, [0, q_len], [48], theta, args[7], 20)
        compare(out[:q_len], num, zs, cnt, "div", "i32", None)
    a = list(args)
    a[5] = torch.tensor([1000], dtype=torch.int32, device="cuda")          # cut to the four pages
    ctx.hccs_attention_cached(*a, **{**kw, "max_kv": 64})
    assert ctx.hccs_device_status() == 16
    num, zs, cnt = orc.attend(args[0][:q_len].cpu().numpy(), c.k, c.v, c.table, [0, q_len], [64], theta, args[7], 20)
    compare(out[:q_len], num, zs, cnt, "div", "i32", None)
    a[5] = torch.tensor([-3], dtype=torch.int32, device="cuda")
    ctx.hccs_attention_cached(*a, **kw)
    assert ctx.hccs_device_status() == 16 and not out[:q_len].any()
    if q_len > 1:
        out.fill_(77)
        ctx.hccs_attention_cached(*args, **{**kw, "max_q": 3})
        assert ctx.hccs_device_status() == 16 and (out[3:] == 77).all() and not (out[:3] == 77).all()
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("q_len", [1, 3])
@pytest.mark.parametrize("d", [64, 128])
def test_the_longest_cache_with_the_largest_sums(hccs, q_len, d):
    """131072 keys, every code -128 and every r 127: sum r V comes within one percent of 2^31.  All scores are equal, so the
    output is the value itself."""
    import torch
    n, hq, hkv, page = 131072, 4, 2, 64
    ctx = hccs.Context(0)
    ctx.hccs_params_upload_wide([(32767, 127, 127), (127 * 127, 127, 127), (32767, 0, 127), (16257, 128 - 1, 127)], n)
    pool = torch.full((n // page, hkv, page, d), -128, dtype=torch.int8, device="cuda")
    table = torch.randperm(n // page, device="cuda").to(torch.int32).view(1, -1)
    Q = torch.full((q_len, hq, d), -128, dtype=torch.int8, device="cuda")
    out = torch.empty((q_len, hq, d), device="cuda")
    ctx.hccs_attention_cached(Q, pool, pool, table, torch.tensor([0, q_len], dtype=torch.int32, device="cuda"),
                              torch.tensor([n], dtype=torch.int32, device="cuda"), out, [3, 3, 3, 3], 20, max_q=q_len, max_kv=n,
                              out_scale=[0.5] * hq, flags=hccs.HCCS_RECIP_REAL)
    assert ctx.hccs_device_status() == 0
    assert (np.abs(_values(out) + 64.0) <= 64.0 * 4 * 2.0 ** -24).all()
    ctx.close()


@pytest.mark.gpu
def test_pools_beyond_four_gigabytes(hccs):
    """The same sequence in the first pages and in the last of pools whose offsets need more than 32 bits."""
    import torch
    rng = np.random.default_rng(21)
    hq, hkv, d, page, pages = 8, 4, 128, 64, 140000          # 4.6 GB each
    ctx = hccs.Context(0)
    ctx.hccs_params_upload_wide(_theta(rng, hq, 300, True), 300)
    kp, vp = (torch.zeros((pages, hkv, page, d), dtype=torch.int8, device="cuda") for _ in range(2))
    low, high = torch.tensor([[2, 0, 4, 1, 3]], dtype=torch.int32, device="cuda"), torch.tensor([[pages - 1, pages - 4, 131072, pages - 2, 139000]], dtype=torch.int32, device="cuda")
    x = torch.randn((300, hq + 2 * hkv, d), device="cuda", dtype=torch.bfloat16)
    pos = torch.arange(300, dtype=torch.int32, device="cuda")
    steps, rope = [np.full(n, 0.03, np.float32) for n in (hq, hkv, hkv)], hccs.hccs_rope_frequencies(d)
    q8 = torch.empty((300, hq, d), dtype=torch.int8, device="cuda")
    got = []
    for table in (low, high):
        slots = table[0].long()[torch.arange(300, device="cuda") // page] * page + torch.arange(300, device="cuda") % page
        ctx.hccs_cache_write(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], q8, kp, vp, pos, slots, *steps, rope=rope)
        back = [torch.empty((300, hkv, d), device="cuda") for _ in range(2)]
        ctx.hccs_cache_read(kp, vp, table, torch.tensor([0, 300], dtype=torch.int32, device="cuda"), *back, *steps[1:], 300)
        outs = []
        for nq in (1, 5):
            out = torch.empty((nq, hq, d), device="cuda")
            ctx.hccs_attention_cached(q8[300 - nq:].contiguous(), kp, vp, table, torch.tensor([0, nq], dtype=torch.int32, device="cuda"),
                                      torch.tensor([300], dtype=torch.int32, device="cuda"), out, [2000] * hq, 20, max_q=nq, max_kv=300,
                                      out_scale=[0.03] * hq, flags=hccs.HCCS_RECIP_REAL)
            outs.append(out)
        got.append(back + outs)
    assert ctx.hccs_device_status() == 0
    for a, b in zip(*got):
        assert a.any() and torch.equal(a, b)
    ctx.close()


@pytest.mark.gpu
def test_calls_on_two_streams_at_once(hccs):
    """Calls of one context on two streams, interleaved, each repeated over its own inputs: they share nothing they write."""
    import torch
    rng = np.random.default_rng(31)
    ctx = hccs.Context(0)
    theta = _theta(rng, 8, 2000, True)
    cases = []
    for q_lens, kv_lens in (([1] * 6, [2000, 900, 1500, 40, 1999, 7]), ([60, 130], [1900, 1000])):
        out, c, (args, kw, _) = attend(hccs, ctx, rng, q_lens, kv_lens, 8, 2, 128, 64, "real", "f32", wide=True, n_design=2000, theta=theta)
        cases.append((args, kw, out.clone(), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for args, kw, want, stream in cases:
            ctx.hccs_attention_cached(*args, **kw, stream=stream)
    torch.cuda.synchronize()
    assert ctx.hccs_device_status() == 0
    for args, kw, want, stream in cases:
        assert torch.equal(args[6], want)
    ctx.close()


@pytest.mark.gpu
def test_nothing_to_see_at_all(hccs):
    """max_kv of zero, no query, no sequence."""
    import torch
    ctx = hccs.Context(0)
    ctx.hccs_params_upload([(300, 3, 85)] * 4, 64)
    pool = torch.zeros((2, 2, 16, 64), dtype=torch.int8, device="cuda")
    table = torch.zeros((2, 1), dtype=torch.int32, device="cuda")
    for nq in (1, 3):
        Q = torch.zeros((2 * nq, 4, 64), dtype=torch.int8, device="cuda")
        out = torch.full((2 * nq, 4, 64), 7, dtype=torch.int32, device="cuda")
        start = torch.tensor([0, nq, 2 * nq], dtype=torch.int32, device="cuda")
        zero = torch.zeros(2, dtype=torch.int32, device="cuda")
        ctx.hccs_attention_cached(Q, pool, pool, table, start, zero, out, [100] * 4, 20, max_q=nq, max_kv=0)
        assert ctx.hccs_device_status() == 0 and not out.any()
        out.fill_(7)
        ctx.hccs_attention_cached(Q, pool, pool, table, torch.zeros_like(start), zero, out, [100] * 4, 20, max_q=nq, max_kv=16)
        assert ctx.hccs_device_status() == 0 and (out == 7).all()
        before = ctx.hccs_launch_count()
        ctx.hccs_attention_cached(Q[:0], pool, pool, table, torch.zeros_like(start), zero, out[:0], [100] * 4, 20, max_q=nq, max_kv=16)
        assert ctx.hccs_launch_count() == before
    ctx.close()


@pytest.mark.gpu
def test_the_first_call_may_be_captured():
    """A fresh process whose first calls of every kernel happen inside a stream capture."""
    import subprocess
    import sys
    code = """
import numpy as np, torch
import paper_2604_02292_b200 as pkg
ctx = pkg.Context(0)
ctx.hccs_params_upload([(300, 3, 85)] * 16, 64)
x = torch.randn(6, 18, 64, device="cuda")
pool = [torch.zeros((4, 1, 16, 64), dtype=torch.int8, device="cuda") for _ in range(2)]
q8 = torch.empty((6, 16, 64), dtype=torch.int8, device="cuda")
table = torch.tensor([[1, 2]], dtype=torch.int32, device="cuda")
slots, pos = torch.arange(16, 22, device="cuda"), torch.arange(6, dtype=torch.int32, device="cuda")
out = [torch.full((n, 16, 64), 7, dtype=torch.int32, device="cuda") for n in (1, 6)]
start = [torch.tensor([0, n], dtype=torch.int32, device="cuda") for n in (1, 6)]
kv = torch.tensor([6], dtype=torch.int32, device="cuda")
back = [torch.full((6, 1, 64), 7.0, device="cuda") for _ in range(2)]
torch.cuda.synchronize()
def calls():
    ctx.hccs_cache_write(x[:, :16], x[:, 16:17], x[:, 17:], q8, *pool, pos, slots, [0.03] * 16, [0.03], [0.03], rope=pkg.hccs_rope_frequencies(64))
    ctx.hccs_attention_cached(q8[5:], *pool, table, start[0], kv, out[0], [3000] * 16, 20, max_q=1, max_kv=32)
    ctx.hccs_attention_cached(q8, *pool, table, start[1], kv, out[1], [3000] * 16, 20, max_q=6, max_kv=32)
    ctx.hccs_cache_read(*pool, table, start[1], *back, [0.03], [0.03], 6)
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    calls()
g.replay()
torch.cuda.synchronize()
got = [t.clone() for t in out + back]
assert not (got[1] == 7).all() and torch.equal(got[0][0], got[1][5])
for t in out + back:
    t.fill_(7)
calls()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, out + back)) and ctx.hccs_device_status() == 0
print("captured")
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=240)
    assert done.returncode == 0 and "captured" in done.stdout, done.stderr[-2000:]


@pytest.mark.gpu
def test_a_run_of_steps(hccs):
    """Generation as a program runs it: a prompt written and attended, then single tokens, then a tree, on another
    stream and through a captured graph; the cache read back at the end."""
    import torch
    rng = np.random.default_rng(11)
    hq, hkv, d, page, B = 6, 3, 64, 16, 2
    ctx = hccs.Context(0)
    theta = _theta(rng, hq, 256, False)
    ctx.hccs_params_upload(theta, 256)
    torch.cuda.synchronize()
    mult = np.full(hq, 3000, np.int32)
    step = [np.full(hq, 0.03, np.float32), np.full(hkv, 0.03, np.float32), np.full(hkv, 0.02, np.float32)]
    rope = hccs.hccs_rope_frequencies(32, 10000.0, interleaved=True)
    pages = 24
    kp, vp = (torch.zeros((pages, hkv, page, d), dtype=torch.int8, device="cuda") for _ in range(2))
    table = torch.from_numpy(rng.permutation(pages)[:B * 10].reshape(B, 10).astype(np.int32)).cuda()
    hk, hv = np.zeros((pages, hkv, page, d), np.int8), np.zeros((pages, hkv, page, d), np.int8)
    lens = [0, 0]
    stream = torch.cuda.Stream()

    def one(q_lens, tree, run):
        nonlocal hk, hv
        T = sum(q_lens)
        x = rng.standard_normal((T, hq + 2 * hkv, d)).astype(np.float32)
        pos = np.concatenate([np.arange(a, a + n) for a, n in zip(lens, q_lens)]).astype(np.int32)
        tab = table.cpu().numpy()
        slots = np.concatenate([[tab[b, j // page] * page + j % page for j in range(lens[b], lens[b] + n)] for b, n in enumerate(q_lens)]).astype(np.int64)
        for b, n in enumerate(q_lens):
            lens[b] += n
        start = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
        got = run(x, pos, slots, start, list(lens), tree, max(q_lens))
        rot = orc.rotate(x, pos, list(rope.freq)[:16], True, 1.0)
        hk = orc.write(hk, orc.quantise(rot[:, hq:hq + hkv], step[1]), slots)
        hv = orc.write(hv, orc.quantise(x[:, hq + hkv:].astype(np.longdouble), step[2]), slots)
        num, zs, cnt = orc.attend(orc.quantise(rot[:, :hq], step[0]), hk, hv, tab, start, lens, theta, mult, 20, tree)
        compare(got, num, zs, cnt, "div", "i32", None)

    def eager(x, pos, slots, start, kv, tree, mq):
        with torch.cuda.stream(stream):
            t = torch.from_numpy(x).cuda()
            q8 = torch.empty((x.shape[0], hq, d), dtype=torch.int8, device="cuda")
            out = torch.empty((x.shape[0], hq, d), dtype=torch.int32, device="cuda")
            ctx.hccs_cache_write(t[:, :hq], t[:, hq:hq + hkv], t[:, hq + hkv:], q8, kp, vp, torch.from_numpy(pos).cuda(),
                                 torch.from_numpy(slots).cuda(), *step, rope=rope)
            ctx.hccs_attention_cached(q8, kp, vp, table, torch.from_numpy(start).cuda(), torch.tensor(kv, dtype=torch.int32).cuda(), out, mult, 20,
                                      max_q=mq, max_kv=160, tree_mask=None if tree is None else torch.from_numpy(tree).cuda())
        stream.synchronize()
        return out

    one([70, 33], None, eager)
    for _ in range(3):
        one([1, 1], None, eager)
    # single tokens from a captured graph, replayed with other inputs
    buf = dict(x=torch.zeros((2, hq + 2 * hkv, d), device="cuda"), pos=torch.zeros(2, dtype=torch.int32, device="cuda"),
               slots=torch.full((2,), -1, dtype=torch.int64, device="cuda"), kv=torch.ones(2, dtype=torch.int32, device="cuda"),
               q8=torch.empty((2, hq, d), dtype=torch.int8, device="cuda"), out=torch.empty((2, hq, d), dtype=torch.int32, device="cuda"),
               start=torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.hccs_cache_write(buf["x"][:, :hq], buf["x"][:, hq:hq + hkv], buf["x"][:, hq + hkv:], buf["q8"], kp, vp, buf["pos"], buf["slots"], *step, rope=rope)
        ctx.hccs_attention_cached(buf["q8"], kp, vp, table, buf["start"], buf["kv"], buf["out"], mult, 20, max_q=1, max_kv=160)

    def replay(x, pos, slots, start, kv, tree, mq):
        buf["x"].copy_(torch.from_numpy(x))
        buf["pos"].copy_(torch.from_numpy(pos))
        buf["slots"].copy_(torch.from_numpy(slots))
        buf["kv"].copy_(torch.tensor(kv, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        return buf["out"]

    for _ in range(3):
        one([1, 1], None, replay)
    one([12, 5], _tree(rng, [12, 5], 1), eager)
    total = sum(lens)
    start = torch.tensor([0, lens[0], total], dtype=torch.int32, device="cuda")
    out = [torch.empty((total, hkv, d), device="cuda") for _ in range(2)]
    ctx.hccs_cache_read(kp, vp, table, start, *out, step[1], step[2], max(lens))
    assert ctx.hccs_device_status() == 0
    tab = table.cpu().numpy()
    for got, pool, st in zip(out, (hk, hv), step[1:]):
        want = np.concatenate([orc.sequence(pool, tab[b], n) for b, n in enumerate(lens)]).astype(np.float32) * st[None, :, None]
        assert (got.cpu().numpy() == want).all()
    ctx.close()


@pytest.mark.gpu
def test_tensors_of_other_kinds_are_refused(hccs):
    """Floats where whole numbers belong, whole numbers where values belong: refused before anything is launched."""
    import torch
    dev = "cuda"
    ctx = hccs.Context(0)
    ctx.hccs_params_upload([(300, 3, 85)] * 2, 64)                        # (a table of the integer modes)
    i8 = lambda *s: torch.zeros(s, dtype=torch.int8, device=dev)          # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=dev)        # noqa: E731
    x, step = torch.zeros((3, 2, 64), device=dev), np.ones(2, np.float32)
    write = dict(q=x, k=x, v=x, q8=i8(3, 2, 64), k_pages=i8(2, 2, 16, 64), v_pages=i8(2, 2, 16, 64), positions=i32(3),
                 slots=torch.arange(3, device=dev), q_step=step, k_step=step, v_step=step)
    read = dict(k_pages=i8(2, 2, 16, 64), v_pages=i8(2, 2, 16, 64), page_table=i32(1, 1), out_start=i32(2), k_out=x.clone(), v_out=x.clone(),
                k_step=step, v_step=step, max_len=3)
    attend = dict(Q=i8(3, 2, 64), k_pages=i8(2, 2, 16, 64), v_pages=i8(2, 2, 16, 64), page_table=i32(1, 1), q_start=i32(2), kv_len=i32(1),
                  O=i32(3, 2, 64), requant_mult=np.ones(2, np.int32), requant_shift=8, max_q=3, max_kv=16, tree_mask=i32(3, 1))
    torch.cuda.synchronize()
    before = ctx.hccs_launch_count()
    f8 = torch.float8_e4m3fn
    for call, args, wrong in [(ctx.hccs_cache_write, write, {"q8": f8, "k_pages": f8, "v_pages": f8, "positions": torch.float32, "slots": torch.float64, "k": torch.float16, "q": torch.int32}),
                              (ctx.hccs_cache_read, read, {"k_pages": f8, "v_pages": f8, "page_table": torch.float32, "out_start": torch.float32, "k_out": torch.int32, "v_out": torch.int16}),
                              (ctx.hccs_attention_cached, attend, {"Q": f8, "k_pages": f8, "v_pages": f8, "page_table": torch.float32, "q_start": torch.float32, "kv_len": torch.float32,
                                                                   "tree_mask": torch.float32, "O": torch.int64})]:
        for name, dtype in wrong.items():
            with pytest.raises((ValueError, hccs.HccsError)):
                call(**{**args, name: args[name].to(dtype)})
    assert ctx.hccs_launch_count() == before
    ctx.hccs_cache_write(**write)
    ctx.hccs_attention_cached(**attend)
    assert ctx.hccs_launch_count() == before + 2
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("rot,interleaved", [(64, False), (32, True), (20, False)])
def test_write_of_far_positions(hccs, rot, interleaved):
    """Angles of up to 2^51 radians: the codes are still those of the angle as it rounds to fp64."""
    import torch
    rng = np.random.default_rng(rot)
    T, d = 257, 64
    x = torch.from_numpy(rng.standard_normal((T, 4, d)).astype(np.float32)).cuda()
    pos = np.concatenate([rng.integers(-2 ** 31, 2 ** 31, T - 6), [2 ** 31 - 1, -2 ** 31, 2 ** 24, 2 ** 24 + 1, 2 ** 24 - 1, 0]]).astype(np.int32)
    freq = [[1.0, 1e6, 0.37, 1000.0, 1e-3][i % 5] * 1.07 ** i for i in range(rot // 2)]
    q8 = torch.zeros((T, 2, d), dtype=torch.int8, device="cuda")
    kp, vp = (torch.zeros((20, 1, 16, d), dtype=torch.int8, device="cuda") for _ in range(2))
    step = [0.02, 0.003]
    ctx = hccs.Context(0)
    ctx.hccs_cache_write(x[:, :2], x[:, 2:3], x[:, 3:], q8, kp, vp, torch.from_numpy(pos).cuda(), torch.arange(T, device="cuda"), step, [0.02], [0.02],
                         rope=hccs.Rope(freq, interleaved=interleaved))
    xs = x.cpu().numpy()
    assert (q8.cpu().numpy() == orc.quantise(orc.rotate(xs[:, :2], pos, freq, interleaved, 1.0), step)).all()
    got = kp.cpu().numpy().transpose(0, 2, 1, 3).reshape(-1, 1, d)[:T]
    assert (got == orc.quantise(orc.rotate(xs[:, 2:3], pos, freq, interleaved, 1.0), [0.02])).all()
    assert ctx.hccs_device_status() == 0
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hkv,d,rot,T", [(1, 0, 128, 128, 5), (1, 0, 64, 64, 3), (0, 1, 128, 128, 2), (3, 0, 128, 96, 17), (1, 1, 64, 2, 33), (0, 2, 64, 34, 9)])
def test_write_of_a_few_heads(hccs, hq, hkv, d, rot, T):
    """Calls so small that a CTA has fewer threads than a head has pairs; queries alone, keys and values alone."""
    import torch
    rng = np.random.default_rng(hq + 10 * hkv + rot)
    x = torch.from_numpy(rng.standard_normal((T, max(hq, 1) + 2 * max(hkv, 1), d)).astype(np.float32)).cuda()
    q, k, v = (x[:, :hq].contiguous() if hq else None), (x[:, hq:hq + hkv].contiguous() if hkv else None), (x[:, hq + hkv:hq + 2 * hkv].contiguous() if hkv else None)
    pos = rng.integers(0, 5000, T).astype(np.int32)
    freq = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
    q8 = torch.zeros((T, hq, d), dtype=torch.int8, device="cuda") if hq else None
    kp, vp = ((torch.zeros((3, hkv, 16, d), dtype=torch.int8, device="cuda") for _ in range(2)) if hkv else (None, None))
    ctx = hccs.Context(0)
    ctx.hccs_cache_write(q, k, v, q8, kp, vp, torch.from_numpy(pos).cuda(), torch.arange(T, device="cuda") if hkv else None,
                         [0.03] * hq if hq else None, [0.03] * hkv if hkv else None, [0.04] * hkv if hkv else None, rope=hccs.Rope(freq))
    xs = x.cpu().numpy()
    if hq:
        assert (q8.cpu().numpy() == orc.quantise(orc.rotate(xs[:, :hq], pos, freq, False, 1.0), [0.03] * hq)).all()
    if hkv:
        back = lambda p: p.cpu().numpy().transpose(0, 2, 1, 3).reshape(-1, hkv, d)[:T]          # noqa: E731
        assert (back(kp) == orc.quantise(orc.rotate(xs[:, hq:hq + hkv], pos, freq, False, 1.0), [0.03] * hkv)).all()
        assert (back(vp) == orc.quantise(xs[:, hq + hkv:hq + 2 * hkv].astype(np.longdouble), [0.04] * hkv)).all()
    assert ctx.hccs_device_status() == 0
    ctx.close()


def _sums_in_64_bits(q, k, v, theta, mult, shift):
    """sum s V and Z of one head's queries q [rows, d] over keys k, v [n, d], exact integers in float64 on the GPU."""
    import torch
    acc = q.double() @ k.double().T
    x = torch.floor((acc * float(mult) + 2.0 ** (shift - 1)) / 2.0 ** shift).clamp(-128, 127)
    big, slope, reach = (float(c) for c in theta)
    s = big - slope * (x.amax(1, keepdim=True) - x).clamp(max=reach)
    return s @ v.double(), s.sum(1, keepdim=True)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [9, 11, 12, 16, 17])
@pytest.mark.parametrize("n", [81952, 100000, 131072])
def test_large_head_groups_on_long_caches(hccs, d, group, n):
    """Single tokens with more than eight query heads per kv head and many keys: against float64, which holds every sum exactly, and bit for
    bit against the kernel for several tokens.  Short sequences under the same bound too."""
    import torch
    rng = np.random.default_rng(n + group)
    page, shift = 64, 20
    ctx = hccs.Context(0)
    theta = _theta(rng, group, n, True)
    ctx.hccs_params_upload_wide(theta, n)
    g = torch.Generator(device="cuda").manual_seed(n + group)
    per = -(-n // page)
    kp, vp = (torch.randint(-128, 128, (per, 1, page, d), device="cuda", generator=g).to(torch.int8) for _ in range(2))
    lens = [n, 300, n // 3, 1]
    table = torch.stack([torch.randperm(per, device="cuda", generator=g) for _ in lens]).to(torch.int32)
    Q = torch.randint(-128, 128, (len(lens), group, d), device="cuda", generator=g).to(torch.int8)
    mult, scale = np.full(group, int(20 / (74.0 ** 2 * math.sqrt(d)) * (1 << shift)), np.int32), rng.uniform(0.01, 0.05, group).astype(np.float32)
    start, kv = torch.arange(len(lens) + 1, dtype=torch.int32, device="cuda"), torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = []
    for max_q in (1, 2):
        out = torch.full((len(lens), group, d), 7.0, device="cuda")
        ctx.hccs_attention_cached(Q, kp, vp, table, start, kv, out, mult, shift, max_q=max_q, max_kv=n, out_scale=scale, flags=hccs.HCCS_RECIP_REAL)
        assert ctx.hccs_device_status() == 0
        got.append(out)
    assert torch.equal(*got)
    for b, length in enumerate(lens):
        pages = table[b, :-(-length // page)].long()
        k, v = (p[pages, 0].reshape(-1, d)[:length] for p in (kp, vp))
        for h in range(group):
            num, z = _sums_in_64_bits(Q[b, h:h + 1], k, v, theta[h], mult[h], shift)
            want = num / z * float(scale[h])
            assert bool(((got[0][b, h].double() - want[0]).abs() <= 4 * 2.0 ** -24 * want[0].abs()).all()), (b, h)
    ctx.close()


@pytest.mark.gpu
def test_captured_calls_outlive_larger_tables(hccs):
    """Uploads of up to 256 heads leave the table where captured launches look for it."""
    import torch
    rng = np.random.default_rng(41)
    ctx = hccs.Context(0)
    runs = []
    theta = _theta(rng, 4, 300, False)
    for q_lens in ([1, 1], [5, 2]):
        out, _, (args, kw, _) = attend(hccs, ctx, rng, q_lens, [300, 40], 4, 2, 64, 16, "real", "f32", n_design=300, theta=theta)
        runs.append((args, kw, out, out.clone()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for args, kw, _, _ in runs:
            ctx.hccs_attention_cached(*args, **kw)
    for heads in (65, 128, 256):
        ctx.hccs_params_upload_wide([(16000, 1, 127)] * heads, 300)
        ctx.hccs_params_upload([(109, 0, 1)] * heads, 300)
    filler = [torch.full((n,), -1, dtype=torch.int32, device="cuda") for n in (256, 1024, 4096)]     # takes what was given back
    ctx.hccs_params_upload(theta, 300)
    for _, _, out, want in runs:
        out.fill_(77)
    graph.replay()
    torch.cuda.synchronize()
    for _, _, out, want in runs:
        assert torch.equal(out, want)
    assert ctx.hccs_device_status() == 0 and all((t == -1).all() for t in filler)
    ctx.close()


def test_first_calls_of_two_threads(binding):
    """The table of integer types is filled on first use: whatever line of that another thread's first call falls on, a right tensor passes.
    For each line of the first look at a tensor, a fresh process in which a second thread makes the same look just before that line."""
    import subprocess
    import sys
    code = """
import os, sys, threading
import torch
from paper_2604_02292_b200 import binding as b

class Fake:                                  # what the binding asks of a tensor on the context's device
    device = torch.device("cuda", 0)
    shape = (4,)
    def __init__(self, dtype): self.dtype = dtype
    def get_device(self): return 0
    def is_contiguous(self): return True
    def element_size(self): return self.dtype.itemsize
    def data_ptr(self): return 4096

ctx = b.Context.__new__(b.Context)
ctx._h, ctx.device = None, 0
failed = []
def look():
    for dtype in (torch.int8, torch.int32, torch.int64):
        try:
            ctx._check(Fake(dtype), "t", dtype.itemsize, (4,))
        except ValueError as e:
            failed.append(str(e))
def first_look(line):
    threads, seen = [], [0]
    def trace(frame, event, arg):
        if not frame.f_code.co_filename.endswith("binding.py"):
            return None
        if event == "line":
            if seen[0] == line:
                threads.append(threading.Thread(target=look))
                threads[0].start()
                threads[0].join(0.1)         # (it may have to wait for this thread)
            seen[0] += 1
        return trace
    sys.settrace(trace)
    look()
    sys.settrace(None)
    for t in threads:
        t.join()
    return 1 if failed else 0 if threads else 2
line = 0
while True:
    child = os.fork()
    if child == 0:
        os._exit(first_look(line))
    result = os.waitstatus_to_exitcode(os.waitpid(child, 0)[1])
    if result == 2:
        break
    assert result == 0, f"a look before line {line} of the first one was refused"
    line += 1
assert line > 0
for dtype, size in ((torch.float32, 4), (torch.bool, 1), (torch.float64, 8)):
    try:
        ctx._check(Fake(dtype), "t", size, (4,))
    except ValueError as e:
        assert "integers" in str(e)
    else:
        raise AssertionError(dtype)
print("passed")
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=240)
    assert done.returncode == 0 and "passed" in done.stdout, done.stderr[-2000:]


@pytest.mark.gpu
@pytest.mark.parametrize("q_len", [1, 4])
def test_scales_of_any_size(hccs, q_len):
    """The real quotient with scales down to the smallest float, and sums Z of 2^26: num and Z to fp32, their quotient with the scale and the
    product round by 2^-24 each; what is subnormal is off by half of its step, 2^-150, besides."""
    rng = np.random.default_rng(51)
    ctx = hccs.Context(0)
    scales = np.array([0.03, 1e-28, -1e-33, 1e-36, 1.1754944e-38, -3e-39, 7e-43, 2.0 ** -149, 2e36, 2.0 ** -60, 2.0 ** -61, 0.0], np.float32)
    hq, n = len(scales), 3001
    theta = np.array([(32767 - 9 * h, int(rng.integers(1, 128)), int(rng.integers(1, 128))) for h in range(hq)], np.int32)
    out, c, (args, kw, _) = attend(hccs, ctx, rng, [q_len], [n], hq, 2, 64, 16, "real", "f32", wide=True, theta=theta, check=False)
    ctx.hccs_attention_cached(*args, **{**kw, "out_scale": scales})
    assert ctx.hccs_device_status() == 0
    num, zs, cnt = orc.attend(args[0][:q_len].cpu().numpy(), c.k, c.v, c.table, [0, q_len], [n], theta, args[7], args[8])
    assert zs.max() > 2 ** 26
    want = num / zs[..., None] * scales.astype(np.float64)[None, :, None]
    off = np.abs(_values(out[:q_len]) - want) - (4.01 * 2.0 ** -24 * np.abs(want) + 2.0 ** -150)
    assert (off <= 0).all(), [(float(scales[h]), float(off[:, h].max())) for h in range(hq) if off[:, h].max() > 0]
    ctx.close()


@pytest.mark.gpu
def test_a_tree_mask_without_words_is_refused(hccs):
    """An empty tensor has no address: it must not pass for no mask, which means causal."""
    import torch
    ctx = hccs.Context(0)
    rng = np.random.default_rng(61)
    for q_len in (1, 3):
        out, _, (args, kw, _) = attend(hccs, ctx, rng, [q_len], [40], 2, 1, 64, 16, "div", "i32")
        out.fill_(77)
        before = ctx.hccs_launch_count()
        with pytest.raises(ValueError, match="tree_mask"):
            ctx.hccs_attention_cached(*args, **{**kw, "tree_mask": torch.empty((out.shape[0], 0), dtype=torch.int32, device="cuda")})
        torch.cuda.synchronize()
        assert ctx.hccs_launch_count() == before and (out == 77).all()
    ctx.close()


@pytest.mark.gpu
def test_page_tables_without_pages(hccs):
    """max_pages of zero, whose table has no address: sequences without keys, and lengths that are cut to none."""
    import torch
    ctx = hccs.Context(0)
    ctx.hccs_params_upload([(300, 3, 85)] * 4, 64)
    pool = torch.full((2, 2, 16, 64), 5, dtype=torch.int8, device="cuda")
    table = torch.empty((2, 0), dtype=torch.int32, device="cuda")
    for nq in (1, 3):
        Q = torch.ones((2 * nq, 4, 64), dtype=torch.int8, device="cuda")
        start = torch.tensor([0, nq, 2 * nq], dtype=torch.int32, device="cuda")
        for length, word in ((0, 0), (9, 16)):
            kv = torch.full((2,), length, dtype=torch.int32, device="cuda")
            out = torch.full((2 * nq, 4, 64), 7, dtype=torch.int32, device="cuda")
            ctx.hccs_attention_cached(Q, pool, pool, table, start, kv, out, [100] * 4, 20, max_q=nq, max_kv=64)
            assert ctx.hccs_device_status() == word and not out.any()
    for starts, word in (([0, 0, 0], 0), ([0, 2, 5], 16)):
        back = [torch.full((6, 2, 64), 7.0, device="cuda") for _ in range(2)]
        ctx.hccs_cache_read(pool, pool, table, torch.tensor(starts, dtype=torch.int32, device="cuda"), *back, [0.1] * 2, [0.1] * 2, 16)
        assert ctx.hccs_device_status() == word and all((t == 7).all() for t in back)
    ctx.close()


def _attend_seen(q, c, row, theta, mult, shift, seen):
    """As the oracle, for one sequence and any pattern: seen [queries, keys]."""
    k, v = (orc.sequence(p, c.table[row], seen.shape[1]).astype(np.int64) for p in (c.k, c.v))
    T, hq, d = q.shape
    num, zs, cnt = np.zeros((T, hq, d), np.int64), np.zeros((T, hq), np.int64), np.zeros((T, hq), np.int64)
    for t in range(T):
        w = seen[t]
        if not w.any():
            continue
        for h in range(hq):
            kh = h // (hq // k.shape[1])
            x = np.clip((k[w, kh] @ q[t, h].astype(np.int64) * int(mult[h]) + (1 << (shift - 1))) >> shift, -128, 127)
            s = theta[h][0] - theta[h][1] * np.minimum(x.max() - x, theta[h][2])
            num[t, h], zs[t, h], cnt[t, h] = s @ v[w, kh], s.sum(), w.sum()
    return num, zs, cnt


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_len", [1, 5, 40])
@pytest.mark.parametrize("tree", [False, True])
def test_bounds_below_the_lengths(hccs, d, q_len, tree):
    """max_kv and max_q below what the sequence has: what is cut is not seen and not computed, the rest is as ever, and both are reported."""
    import torch
    rng = np.random.default_rng(71)
    ctx = hccs.Context(0)
    n = 700
    mask = None
    if tree:                                               # any bits, those of nodes beyond the bounds among them
        mask = rng.integers(0, 2 ** 32, (q_len, 2), dtype=np.uint64).astype(np.uint32).view(np.int32)
    out, c, (args, kw, theta) = attend(hccs, ctx, rng, [q_len], [n], 4, 2, d, 16, "div", "i32", n_design=n, tree=mask)
    q = args[0][:q_len].cpu().numpy()

    def check(max_q, max_kv):
        rows = min(q_len, max_q)
        seen = np.zeros((rows, n), bool)
        for t in range(rows):
            for j in range(min(n, max_kv)):
                new = j - (n - q_len)
                seen[t, j] = new < 0 or (new <= t if mask is None else new < max_q and bool((int(mask[t, new // 32]) >> (new % 32)) & 1))
        out.fill_(77)
        ctx.hccs_attention_cached(*args, **{**kw, "max_q": max_q, "max_kv": max_kv})
        assert ctx.hccs_device_status() == (16 if max_kv < n or max_q < q_len else 0), (max_q, max_kv)
        compare(out[:rows], *_attend_seen(q[:rows], c, 0, theta, args[7], args[8], seen), "div", "i32", None)
        assert (out[rows:] == 77).all()
    for max_kv in (0, 1, 16, 127, 128, 129, 500, n - q_len, n - 1, n):
        check(q_len, max_kv)
    for max_q in (1, 2, 4, 31, 32, 33):
        if max_q < q_len:
            check(max_q, n)
            check(max_q, n - q_len + 1)
    ctx.close()


@pytest.mark.gpu
@pytest.mark.parametrize("max_q", [1, 4])
def test_starts_that_fall_or_leave_the_tokens(hccs, max_q):
    """q_start is cut to the tokens; a sequence whose start lies behind its end has none."""
    import torch
    rng = np.random.default_rng(81)
    ctx = hccs.Context(0)
    T, lens = 8, [50, 40, 30, 20]
    out, c, (args, kw, theta) = attend(hccs, ctx, rng, [2] * 4, lens, 4, 2, 64, 16, "real", "f32")
    for starts, owners in (([5, 3, 6, 99, 99], {1: (3, 6), 2: (6, 8)}), ([-9, 2, 2, 7, 2 ** 31 - 1], {0: (0, 2), 2: (2, 7), 3: (7, 8)}),
                           ([-2 ** 31, -1, 0, 1, 0], {2: (0, 1)})):
        big = torch.full((T + 6, 4, 64), 77.0, device="cuda")
        o = big[3:3 + T]
        a = list(args)
        a[0], a[4], a[6] = args[0][:T], torch.tensor(starts, dtype=torch.int32, device="cuda"), o
        ctx.hccs_attention_cached(*a, **{**kw, "max_q": max_q})
        ctx.hccs_device_status()
        done = np.zeros(T, bool)
        for b, (s0, s1) in owners.items():
            rows = min(s1 - s0, max_q)
            seen = np.arange(lens[b])[None, :] <= (lens[b] - (s1 - s0)) + np.arange(rows)[:, None]
            sums = _attend_seen(args[0][s0:s0 + rows].cpu().numpy(), c, b, theta, args[7], args[8], seen)
            compare(o[s0:s0 + rows], *sums, "real", "f32", kw["out_scale"])
            done[s0:s0 + rows] = True
        assert (o[torch.from_numpy(~done).cuda()] == 77).all() and (big[:3] == 77).all() and (big[3 + T:] == 77).all()
    ctx.close()
