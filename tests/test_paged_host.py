"""CPU-only tests of the paged cache, of attention over it and of the verification of drafted tokens: exported symbols, refusals found on the host (no GPU is touched: every call here fails, or
has nothing to do, before any launch), and the oracles against closed forms."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20  # an address that is never used


@pytest.fixture(scope="module")
def ca():
    import paper_2509_21275_amd as ca
    if not os.path.exists(ca.LIB_PATH):
        from paper_2509_21275_amd.build import build_library
        build_library()
    return ca


def test_library_exports_what_the_headers_declare(ca):
    names = set()
    for h in ("paged_cache.h", "paged_attn.h", "draft_verify.h"):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", h)).read(), flags=re.S)
        names |= set(re.findall(r"\bint ((?:paged_cache|paged_attn|draft_verify)[a-z0-9_]*)\s*\(", text))
    assert {"paged_cache_validate", "paged_cache_workspace_bytes", "paged_cache_extend", "paged_cache_truncate", "paged_cache_write", "paged_attn_validate",
            "paged_attn_workspace_bytes", "paged_attn_fwd", "draft_verify_workspace_bytes", "draft_verify"} == names
    lib = ctypes.CDLL(ca.LIB_PATH)
    assert all(hasattr(lib, n) for n in names)


def test_table_refusals(ca):
    from paper_2509_21275_amd import paged_cache as pc
    pc._bind()
    lib = ca._lib
    assert pc.paged_cache_validate(pc.make_desc(1, 1, 1, 1)) == ca.OK and pc.paged_cache_validate(pc.make_desc(65536, 32767, 65536, 2**31 - 1)) == ca.OK
    for d in ((0, 4, 16, 8), (-1, 4, 16, 8), (4, 0, 16, 8), (4, 4, 0, 8), (4, 4, 16, 0), (4, 32768, 65536, 8)):
        assert pc.paged_cache_validate(pc.make_desc(*d)) == ca.INVALID_ARG, d
    for d in ((65537, 4, 16, 8), (4, 4, 65537, 8)):
        assert pc.paged_cache_validate(pc.make_desc(*d)) == ca.UNSUPPORTED, d
    assert lib.paged_cache_validate(None) == ca.INVALID_ARG
    desc = pc.make_desc(4, 4, 16, 8)
    size = pc.paged_cache_workspace_bytes(desc)
    names = ("new", "kv_len", "held", "table", "free", "num_free", "kv_len_out", "held_out", "num_free_out")

    def extend(d=desc, q_start=P, slots=P, rows=8, granted=P, ws=P, size=size, **kw):
        return lib.paged_cache_extend(ctypes.byref(d), *[kw.get(n, P) for n in names], q_start, slots, rows, granted, ws, size, None)

    def truncate(d=desc, ws=P, size=size, **kw):
        return lib.paged_cache_truncate(ctypes.byref(d), *[kw.get(n, P) for n in names], ws, size, None)

    for call in (extend, truncate):
        for n in names:
            assert call(**{n: None}) == ca.INVALID_ARG and call(**{n: P + 2}) == ca.INVALID_ARG, n
        assert call(ws=None) == ca.INVALID_ARG and call(ws=P + 128) == ca.INVALID_ARG and call(size=size - 1) == ca.WORKSPACE_TOO_SMALL
        assert call(d=pc.make_desc(0, 4, 16, 8)) == ca.INVALID_ARG
    for kw in (dict(q_start=None), dict(q_start=P + 1), dict(slots=None), dict(slots=P + 4), dict(rows=-1), dict(granted=P + 2)):
        assert extend(**kw) == ca.INVALID_ARG, kw
    with pytest.raises(ValueError):
        pc.paged_cache_extend(desc, *[None] * 13)
    with pytest.raises(ValueError):
        pc.paged_cache_truncate(desc, *[None] * 10)


def test_write_refusals(ca):
    from paper_2509_21275_amd import paged_cache as pc
    pc._bind()

    def write(rows=4, H=2, d=64, page=16, pages=8, kind=0, k=P, ks=128, v=P, vs=128, slots=P, k_scale=P, v_scale=P, kc=P, vc=P):
        return ca._lib.paged_cache_write(rows, H, d, page, pages, kind, k, ks, v, vs, slots, k_scale, v_scale, kc, vc, None)

    for kw in (dict(rows=-1), dict(H=0), dict(page=0), dict(pages=0), dict(kind=2), dict(kind=-1), dict(k=None), dict(k=P + 1), dict(ks=127), dict(v=None), dict(vs=0), dict(slots=None),
               dict(slots=P + 4), dict(kc=None), dict(kc=P + 8), dict(vc=P + 2), dict(kind=1, k_scale=None), dict(kind=1, v_scale=P + 2), dict(rows=2**31 - 1, H=16384, ks=2**30, vs=2**30)):
        assert write(**kw) == ca.INVALID_ARG, kw
    assert write(d=80) == ca.UNSUPPORTED and write(H=16385) == ca.UNSUPPORTED and write(page=65537) == ca.UNSUPPORTED and write(rows=0, k=None) == ca.OK
    with pytest.raises(ValueError):
        pc.paged_cache_write(None, None, None, None, None)


def test_write_refuses_more_than_a_launch_has_threads_for(ca):
    """A thread to eight elements, and below 2^32 threads: 2^35 - 2^11 elements are the most, as the header says."""
    from paper_2509_21275_amd import paged_cache as pc
    pc._bind()
    text = open(os.path.join(ROOT, "include", "paged_cache.h")).read()
    assert "rows * num_kv_heads * head_dim <= 2^35 - 2^11" in text
    for rows, heads, dim in ((2**28, 1, 128), (2**28 - 15, 2, 64), (2**20, 256, 128), (2**21 - 1, 257, 64)):
        assert rows * heads * dim > 2**35 - 2**11
        assert ca._lib.paged_cache_write(rows, heads, dim, 16, 1000, 0, P, heads * dim, P, heads * dim, P, None, None, P, P, None) == ca.INVALID_ARG


def test_attention_refusals(ca):
    from paper_2509_21275_amd import paged_attn as pa
    pa._bind()
    base = dict(num_q_heads=8, num_kv_heads=2, head_dim=64, num_seqs=4, total_q=5, page_size=16, num_pages=32, max_pages=8, softmax_scale=0.1)

    def desc(**kw):
        return pa.make_desc(**{**base, **kw})

    assert pa.paged_attn_validate(desc()) == ca.OK
    for kw in (dict(num_q_heads=0), dict(num_kv_heads=0), dict(num_seqs=0), dict(total_q=-1), dict(page_size=0), dict(num_pages=0), dict(max_pages=0), dict(softmax_scale=0.0),
               dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")), dict(softmax_scale=-1.0), dict(total_q=2**28), dict(max_pages=2**27), dict(num_pages=2**26)):
        assert pa.paged_attn_validate(desc(**kw)) == ca.INVALID_ARG, kw
    for kw in (dict(head_dim=80), dict(head_dim=32), dict(num_q_heads=9), dict(num_q_heads=32768), dict(num_seqs=65537), dict(page_size=65537)):
        assert pa.paged_attn_validate(desc(**kw)) == ca.UNSUPPORTED, kw
    # 4096 sequences, a row to each, of up to 2^25 tokens: 2^30 blocks of 128 keys
    most = dict(num_q_heads=2, num_seqs=4096, total_q=4096)
    assert pa.paged_attn_validate(desc(max_pages=2**21, **most)) == ca.OK and pa.paged_attn_validate(desc(max_pages=2**21 + 1, **most)) == ca.INVALID_ARG
    bad = desc()
    bad.cache_type = 2
    assert pa.paged_attn_validate(bad) == ca.INVALID_ARG and ca._lib.paged_attn_validate(None) == ca.INVALID_ARG
    with pytest.raises(ValueError):
        desc(cache_type="fp16")
    size = pa.paged_attn_workspace_bytes(desc())

    def fwd(d=None, q=P, qs=512, k=P, v=P, k_scale=P, v_scale=P, table=P, kv_len=P, q_start=P, o=P, os_=512, lse=P, ws=P, size=size):
        return ca._lib.paged_attn_fwd(ctypes.byref(d or desc()), q, qs, k, v, k_scale, v_scale, table, kv_len, q_start, o, os_, lse, ws, size, None)

    for kw in (dict(q=None), dict(q=P + 1), dict(qs=511), dict(k=None), dict(k=P + 8), dict(v=None), dict(v=P + 2), dict(table=None), dict(table=P + 2), dict(kv_len=None),
               dict(kv_len=P + 1), dict(q_start=None), dict(o=None), dict(o=P + 1), dict(os_=0), dict(lse=P + 2), dict(ws=None), dict(ws=P + 16)):
        assert fwd(**kw) == ca.INVALID_ARG, kw
    eight = desc(cache_type="e4m3")
    assert fwd(eight, k_scale=None) == ca.INVALID_ARG and fwd(eight, v_scale=P + 1) == ca.INVALID_ARG
    assert fwd(size=size - 1) == ca.WORKSPACE_TOO_SMALL and fwd(desc(total_q=0), q=None, ws=None) == ca.OK
    with pytest.raises(ValueError):
        pa.paged_attn_fwd(desc(), *[None] * 9)


def test_verify_refusals(ca):
    from paper_2509_21275_amd import draft_verify as dv
    size = dv.draft_verify_workspace_bytes(4, 3, 1000)

    def run(batch=4, K=3, V=1000, f32=1, target=P, ts=1000, draft=P, ds=1000, tokens=P, count=P, u=P, last=P, accepted=P, rejected=P, out=P, ws=P, size=size):
        return ca._lib.draft_verify(batch, K, V, f32, target, ts, draft, ds, tokens, count, u, last, accepted, rejected, out, ws, size, None)

    for kw in (dict(batch=-1), dict(K=-1), dict(V=0), dict(target=None), dict(target=P + 2), dict(ts=999), dict(draft=P + 2), dict(ds=0), dict(tokens=None), dict(tokens=P + 2),
               dict(count=P + 1), dict(u=None), dict(u=P + 2), dict(last=None), dict(last=P + 1), dict(accepted=None), dict(accepted=P + 2), dict(rejected=P + 1), dict(out=None),
               dict(out=P + 2), dict(ws=None), dict(ws=P + 8), dict(f32=0, target=P + 1), dict(batch=2**20, V=2**18), dict(batch=2**23, V=10)):
        assert run(**kw) == ca.INVALID_ARG, kw
    assert run(K=65) == ca.UNSUPPORTED and run(V=2**24 + 1, ts=2**25, ds=2**25) == ca.UNSUPPORTED
    assert run(size=size - 1) == ca.WORKSPACE_TOO_SMALL and run(batch=0, target=None, ws=None) == ca.OK
    for args in ((-1, 1, 1), (1, -1, 1), (1, 1, 0)):
        with pytest.raises(ca.ChunkAttnError) as e:
            dv.draft_verify_workspace_bytes(*args)
        assert e.value.code == ca.INVALID_ARG
    with pytest.raises(ValueError):
        dv.draft_verify(*[None] * 10)


# ---- the oracles ----
def test_oracle_of_the_tables():
    from oracle import paged_oracle as orc
    table = np.full((3, 4), -1)
    table[0, 0] = 9
    stack = np.array([5, 6, 7, 8, 0, 0, 0, 0, 0, 0])
    kv_len, held, t, free, q_start, slots, granted = orc.extend(4, 10, [3, 9, 2], np.array([3, 0, 0]), np.array([1, 0, 0]), table, stack, 4, 20)
    # the first takes page 8 for its tokens 4 and 5; the second has use for three pages, all that are left; the third finds none
    assert t[0].tolist() == [9, 8, -1, -1] and t[1].tolist() == [7, 6, 5, -1] and free == 0 and granted.tolist() == [1, 1, 0]
    assert slots[:14].tolist() == [39, 32, 33, 28, 29, 30, 31, 24, 25, 26, 27, 20, -1, -1] and q_start.tolist() == [0, 3, 12, 14]
    kv_len, held, s, free = orc.truncate(4, [0, 5, 9], kv_len, held, t, stack, free)
    assert kv_len.tolist() == [6, 4, 0] and held.tolist() == [2, 1, 0] and s[:free].tolist() == [6, 5]


def test_oracle_of_the_attention():
    from oracle import paged_oracle as orc
    rng = np.random.default_rng(0)
    k, v, q = rng.normal(size=(5, 1, 2, 64)), rng.normal(size=(5, 1, 2, 64)), rng.normal(size=(2, 2, 64))
    table, order = np.array([[3, 0, 4]]), [(3, 0), (3, 1), (0, 0), (0, 1), (4, 0)]
    for row, o, lse, *_ in orc.attention(q, k, v, table, [5], [0, 2], 0.125):
        ks, vs = (np.array([c[p, 0, r] for p, r in order[:4 + row]]) for c in (k, v))
        w = np.exp(q[row] @ ks.T * 0.125)
        assert np.allclose(o, w / w.sum(-1, keepdims=True) @ vs) and np.allclose(lse, np.log(w.sum(-1)))
    zero = list(orc.attention(q, k * 0, v, table, [5], [0, 1], 0.125))[0]
    assert np.allclose(zero[1][0], np.mean([v[p, 0, r] for p, r in order], 0)) and np.allclose(zero[2], np.log(5))


def test_oracle_of_the_verification_draws_as_the_target():
    """Over all random numbers of a grid the first token is distributed as the target's probabilities, whatever the draft's."""
    from oracle import paged_oracle as orc
    p, q = np.array([[0.5, 0.25, 0.25, 0.0], [0.25] * 4]), np.array([[0.125, 0.5, 0.25, 0.125]])
    got = np.zeros(4)
    m = 32
    for d in range(4):
        for i in range(m):
            for j in range(m):
                kept, out = orc.verify(p, q, [d], 1, [(i + 0.5) / m], (j + 0.5) / m)
                got[out[0]] += q[0, d] / m / m
    assert np.allclose(got, p[0])


# ---- the division of the attention's work ----
@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_division_of_work_in_any_numbers(tmp_path):
    exe = str(tmp_path / "paged_shares")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", os.path.join(ROOT, "tests", "native", "paged_shares.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout[-2000:]


@pytest.mark.parametrize("heads", [1, 3, 5, 8, 10, 12, 24, 40, 96, 200, 255, 256, 257, 300, 512, 600])
def test_no_more_workgroups_than_fit_at_once(ca, heads):
    """Two workgroups to each of 256 compute units: shares of all heads, by the parts that the workspace has room for, are no more, but for more heads than half of that."""
    from paper_2509_21275_amd import paged_attn as pa
    size = pa.paged_attn_workspace_bytes(pa.make_desc(heads, heads, 128, 8, 8, 16, 4096, 512, 0.1))
    shares, rest = divmod(size, 2 * heads * 32 * 130 * 4 + 16)
    assert rest == 0 and shares == (512 // heads if heads <= 256 else 2 if heads < 512 else 1)
