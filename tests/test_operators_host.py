"""CPU-only tests of the operators around chunk attention: exported symbols, the frequencies, and refusals found on the host (no GPU is touched: every call
here fails, or has nothing to do, before any launch)."""
import ctypes
import os
import re

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ca():
    import paper_2509_21275_amd as ca
    if not os.path.exists(ca.LIB_PATH):
        from paper_2509_21275_amd.build import build_library
        build_library()
    return ca


def test_library_exports_what_the_headers_declare(ca):
    names = set()
    for h in ("chunk_rope.h", "fused_norm.h", "chunk_linear.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", h)).read(), flags=re.S)
        names |= set(re.findall(r"\bint ((?:chunk_rope|fused_norm|chunk_linear)_[a-z0-9_]+)\s*\(", text))
    assert {"chunk_rope_frequencies", "chunk_rope_fwd", "chunk_rope_bwd", "fused_norm_fwd", "fused_norm_bwd", "fused_norm_bwd_workspace_bytes",
            "chunk_linear_validate", "chunk_linear_workspace_bytes", "chunk_linear_fwd", "chunk_linear_bwd", "chunk_linear_step"} == names
    lib = ctypes.CDLL(ca.LIB_PATH)
    assert all(hasattr(lib, n) for n in names)


@pytest.mark.parametrize("kw", [dict(), dict(base=500000.0), dict(scaling="linear", factor=4.0), dict(scaling="base", factor=4.5),
                                dict(scaling="ramp", factor=8.0, original_length=8192, low_rotations=1.0, high_rotations=4.0)])
@pytest.mark.parametrize("rotary", [2, 38, 64, 128, 256])
def test_frequencies(ca, rotary, kw):
    from oracle import rope_oracle as orc
    from paper_2509_21275_amd import chunk_rope as cr
    if rotary == 2 and kw.get("scaling") == "base":
        pytest.skip("one pair has no last frequency to divide")
    want = orc.frequencies(rotary, kw.get("base", 10000.0), kw.get("scaling", "none"), kw.get("factor", 1.0), kw.get("original_length", 0),
                           kw.get("low_rotations", 1.0), kw.get("high_rotations", 32.0))
    assert np.allclose(cr.rope_frequencies(rotary, **kw), want, rtol=1e-13, atol=0)  # a few units of float64 in each power
    if kw.get("scaling") == "base":
        plain = orc.frequencies(rotary)
        assert want[0] == plain[0] and abs(want[-1] * 4.5 / plain[-1] - 1) < 1e-12


@pytest.mark.parametrize("kw", [dict(rotary_dim=3), dict(rotary_dim=0), dict(rotary_dim=-2), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")),
                                dict(factor=0.5), dict(factor=float("nan")), dict(scaling="ramp"), dict(scaling="ramp", original_length=float("nan")),
                                dict(scaling="ramp", original_length=10, low_rotations=4.0, high_rotations=4.0), dict(rotary_dim=2, scaling="base")])
def test_frequencies_refused(ca, kw):
    from paper_2509_21275_amd import chunk_rope as cr
    with pytest.raises(ca.ChunkAttnError) as e:
        cr.rope_frequencies(**{"rotary_dim": 64, **kw})
    assert e.value.code == ca.INVALID_ARG


def test_rope_refusals(ca):
    from paper_2509_21275_amd import chunk_rope as cr
    cr._bind()
    lib, P = ca._lib, 1 << 20  # an address that is never used

    def fwd(rope=None, segs=((0, 8, 0, 8),), d=128, q=P, qs=8 * 128, k=P, ks=2 * 128, qo=2 * P, qos=8 * 128, ko=2 * P, kos=2 * 128, total_kv=16):
        desc = ca.make_desc(segs, 8, 2, d, segs[-1][0] + segs[-1][1], total_kv, 0.1)
        return lib.chunk_rope_fwd(ctypes.byref(desc), ctypes.byref(rope or cr.make_rope(d)), q, qs, k, ks, qo, qos, ko, kos, None)

    bad = cr.make_rope(64)
    for field, value in (("rotary_dim", 63), ("rotary_dim", 0), ("rotary_dim", 130), ("magnitude", float("nan")), ("magnitude", float("inf"))):
        r = cr.make_rope(128)
        setattr(r, field, value)
        assert fwd(r) == ca.INVALID_ARG, (field, value)
    assert fwd(cr.make_rope(128, frequencies=[float("nan")] * 64)) == ca.INVALID_ARG
    assert fwd(cr.make_rope(128, frequencies=[1.0] * 63 + [float("inf")])) == ca.INVALID_ARG
    bad.frequencies = None
    assert fwd(bad) == ca.INVALID_ARG
    assert fwd(segs=((1, 8, 0, 8),)) == ca.BAD_SEGMENT and fwd(d=80) == ca.UNSUPPORTED
    for kw in (dict(qs=1023), dict(ks=255), dict(qos=1000), dict(kos=0), dict(q=None), dict(qo=None), dict(ko=None), dict(q=P + 1), dict(ko=P + 1),
               dict(qo=P, qos=2000), dict(ko=P, kos=512), dict(ko=P, segs=((0, 8, 0, 10),))):
        assert fwd(**kw) == ca.INVALID_ARG, kw
    assert fwd(q=None, qo=None, k=None, ko=None) == ca.OK  # nothing to do
    desc = ca.make_desc([(0, 8, 0, 8)], 8, 2, 128, 8, 8, 0.1)
    assert lib.chunk_rope_bwd(ctypes.byref(desc), ctypes.byref(cr.make_rope(128)), None, 0, P, 256, 1, None, 0, P, 256, None) == ca.INVALID_ARG  # float32 in place
    assert lib.chunk_rope_bwd(ctypes.byref(desc), ctypes.byref(cr.make_rope(128)), None, 0, P + 2, 256, 1, None, 0, 2 * P, 256, None) == ca.INVALID_ARG
    with pytest.raises(ValueError):
        cr.make_rope(64, frequencies=[1.0])


def test_norm_refusals(ca):
    from paper_2509_21275_amd import fused_norm as fn
    fn._bind()
    lib, P = ca._lib, 1 << 20

    def desc(**kw):
        base = dict(rows=4, cols=64, eps=1e-5, residual_scale=1.0, block_scale=1.0, y=P, y_stride=64, gate=P, gate_stride=64, residual=P, residual_stride=64,
                    post_weight=P, pre_weight=P)
        return fn.Norm(**{**base, **kw})

    def fwd(out=2 * P, out_stride=64, h=3 * P, h_stride=64, **kw):
        return lib.fused_norm_fwd(ctypes.byref(desc(**kw)), out, out_stride, h, h_stride, None)

    def bwd(stored=P, d_out=P, d_h=P, dy=P, dg=P, dr=P, dpost=P, dpre=P, ws=P, size=1 << 20, stride=64, **kw):
        return lib.fused_norm_bwd(ctypes.byref(desc(**kw)), stored, stride, d_out, stride, d_h, stride, dy, stride, dg, stride, dr, stride, dpost, dpre, 0, ws, size, None)

    for call in (fwd, bwd):
        assert call(cols=16385, y_stride=16385, gate_stride=16385, residual_stride=16385) == ca.UNSUPPORTED
        for kw in (dict(rows=-1), dict(cols=0), dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(residual_scale=float("nan")),
                   dict(block_scale=float("inf")), dict(gate_kind=3), dict(gate_kind=-1), dict(y=None), dict(y_stride=63), dict(gate_stride=1), dict(residual_stride=0),
                   dict(y=P + 1), dict(post_weight=P + 1), dict(weight_is_f32=1, pre_weight=P + 2), dict(residual_is_f32=1, residual=P + 2)):
            assert call(**kw) == ca.INVALID_ARG, kw
    for kw in (dict(h=None), dict(pre_weight=None), dict(out=None, h=None, pre_weight=None), dict(out_stride=63), dict(h_stride=63),
               dict(y=None, gate=None, post_weight=None, residual=None)):
        assert fwd(**kw) == ca.INVALID_ARG, kw
    for kw in (dict(stored=None), dict(d_h=None), dict(d_out=None, d_h=None, pre_weight=None, dpre=None), dict(pre_weight=None), dict(post_weight=None),
               dict(gate=None), dict(ws=None), dict(ws=P + 8), dict(stride=63), dict(dpost=P + 2), dict(dy=P + 1)):
        assert bwd(**kw) == ca.INVALID_ARG, kw
    assert bwd(size=fn.fused_norm_bwd_workspace_bytes(4, 64) - 1) == ca.WORKSPACE_TOO_SMALL
    assert fwd(rows=0) == ca.OK
    for args in ((-1, 64), (4, 0)):
        with pytest.raises(ca.ChunkAttnError):
            fn.fused_norm_bwd_workspace_bytes(*args)
    with pytest.raises(ca.ChunkAttnError) as e:
        fn.fused_norm_bwd_workspace_bytes(4, 16385)
    assert e.value.code == ca.UNSUPPORTED
    with pytest.raises(ValueError):
        fn.fused_norm_fwd(None, None, None, None, None, None, None)


def test_linear_refusals(ca):
    from paper_2509_21275_amd import chunk_linear as cl
    cl._bind()
    lib, P = ca._lib, 1 << 20

    def desc(segs=((0, 8, -1, -1),), H=4, Hk=2, d=64, total=8, states=2, scale=0.1):
        return cl.make_desc(segs, H, Hk, d, total, states, scale)

    ok = [((0, 8, -1, -1),), ((1, 2, 0, 1), (5, 3, 0, 0)), ((0, 1, -1, -1), (1, 1, -1, -1))]
    assert all(cl.chunk_linear_validate(desc(s)) == ca.OK for s in ok)
    for kw in (dict(H=0), dict(Hk=0), dict(total=0), dict(states=-1), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(segs=())):
        assert cl.chunk_linear_validate(desc(**kw)) == ca.INVALID_ARG, kw
    for kw in (dict(d=80), dict(d=32), dict(H=3), dict(H=16386)):
        assert cl.chunk_linear_validate(desc(**kw)) == ca.UNSUPPORTED, kw
    for segs in (((0, 0, -1, -1),), ((0, 9, -1, -1),), ((-1, 3, -1, -1),), ((0, 4, -1, -1), (3, 2, -1, -1)), ((4, 2, -1, -1), (0, 2, -1, -1)), ((0, 8, 2, -1),),
                 ((0, 8, -2, -1),), ((0, 8, -1, 2),), ((0, 4, -1, 1), (4, 4, -1, 1)), ((1, 2**31 - 1, -1, -1),)):
        assert cl.chunk_linear_validate(desc(segs)) == ca.BAD_SEGMENT, segs
    assert lib.chunk_linear_validate(None) == ca.INVALID_ARG

    def fwd(d, q=P, lg=P, s_in=P, o=P, s_out=2 * P, ws=P, size=1 << 40):
        return lib.chunk_linear_fwd(ctypes.byref(d), q, P, P, lg, s_in, o, s_out, ws, size, None)

    def bwd(d, q=P, s_in=P, ds_out=3 * P, dv=P, ds_in=2 * P, ws=P, size=1 << 40):
        return lib.chunk_linear_bwd(ctypes.byref(d), q, P, P, P, s_in, P, ds_out, P, P, dv, ds_in, ws, size, None)

    one, long = desc(((0, 8, 0, 1),)), desc(((0, 5000, 0, 1),), total=5000)
    f, b = cl.chunk_linear_workspace_bytes(long)
    assert b >= f > 0 and cl.chunk_linear_workspace_bytes(one) == (0, 0)
    for kw in (dict(q=None), dict(q=P + 8), dict(lg=None), dict(lg=P + 2), dict(o=None), dict(s_in=None), dict(s_out=None), dict(s_in=P + 4)):
        assert fwd(one, **kw) == ca.INVALID_ARG, kw
    for kw in (dict(q=None), dict(dv=P + 2), dict(s_in=None), dict(ds_in=P + 8)):
        assert bwd(one, **kw) == ca.INVALID_ARG, kw
    for call, size in ((fwd, f), (bwd, b)):
        assert call(long, ws=None) == ca.INVALID_ARG and call(long, ws=P + 128) == ca.INVALID_ARG
        assert call(long, size=size - 1) == ca.WORKSPACE_TOO_SMALL
    # slots in place: one segment's state_out may not be another's state_in; and a gradient goes to one place only
    crossed, shared = desc(((0, 4, 0, 1), (4, 4, 1, -1))), desc(((0, 4, 0, -1), (4, 4, 0, 1)))
    assert fwd(crossed, s_out=P) == ca.BAD_SEGMENT and bwd(crossed, ds_in=3 * P) == ca.BAD_SEGMENT and bwd(shared) == ca.BAD_SEGMENT

    def step(B=4, H=4, Hk=2, d=64, q=P, s_in=P, s_out=P, n=4, slots=P, o=P, scale=0.1):
        return lib.chunk_linear_step(B, H, Hk, d, q, P, P, P, s_in, s_out, n, slots, o, scale, None)

    for kw in (dict(B=-1), dict(H=0), dict(n=-1), dict(scale=float("nan")), dict(scale=-1.0), dict(q=None), dict(s_in=None), dict(s_out=P + 4), dict(slots=P + 2),
               dict(slots=None), dict(o=P + 2), dict(B=2**31 - 1)):
        assert step(**kw) == ca.INVALID_ARG, kw
    assert step(d=80) == ca.UNSUPPORTED and step(H=3) == ca.UNSUPPORTED and step(B=0) == ca.OK
