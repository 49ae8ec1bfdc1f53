"""Refusals of the cache's C entry points, found on the host before any launch.  No GPU: every call fails validation or has nothing to
do."""
import ctypes as C

import pytest

from paper_2302_12510_amd import binding as B

P, ODD = 0x1000, 0x1004                                  # never dereferenced


def heads(n=4, h=2, d=64, type=0, data=P, stride=None):
    return B.Heads(data, n, h * d if stride is None else stride, d, h, d, type)


def cache(pages=8, h=2, page=16, d=64, kb=8, vb=4, layers=1, **at):
    p = [at.get(n, P) for n in ("k_codes", "k_scales", "v_codes", "v_scales")]
    return B.KVCacheStruct(*p, layers, pages, h, page, d, B.fmt(kb, True), B.fmt(vb, at.get("v_signed", True)))


NONE = B.KVPrefixStruct()


def norm(q=None, k=None, wq=P, wk=P, pos=P, cos=P, sin=P, rows=10, rotary=64, neighbours=0, eps=1e-6, qo=None, ko=None):
    q, k = q or heads(), k or heads(h=1)
    return B.lib().dybit_head_norm_rope(q, k, wq, wk, pos, cos, sin, rows, rotary, neighbours, eps, qo or q, ko or k, None)


def test_norm():
    assert norm(q=heads(n=0), k=heads(n=0, h=1)) == B.OK
    assert norm(q=heads(data=None)) == B.ERR_NULL
    assert norm(wq=None) == norm(wk=None) == norm(pos=None) == norm(cos=None) == norm(sin=None) == B.ERR_NULL
    assert norm(q=heads(data=0x1001)) == B.ERR_ALIGNMENT
    assert norm(q=heads(type=3)) == norm(k=heads(h=1, type=1)) == norm(k=heads(n=3, h=1)) == norm(k=heads(h=1, d=32)) == B.ERR_INVALID_ARG
    assert norm(qo=heads(h=3)) == norm(qo=heads(type=1)) == B.ERR_INVALID_ARG
    assert norm(rotary=0) == norm(rotary=3) == norm(rotary=66) == norm(neighbours=2) == norm(eps=-1.0) == norm(eps=float("nan")) == norm(rows=-1) == B.ERR_INVALID_ARG
    assert norm(q=heads(d=63), k=heads(h=1, d=63), rotary=2) == norm(q=heads(d=514), k=heads(h=1, d=514)) == B.ERR_INVALID_ARG


def test_norm_gradient():
    L, q, k = B.lib(), heads(), heads(h=1)
    call = lambda dwq=P, dwk=P, work=P, g=q: L.dybit_head_norm_rope_bwd(g, k, q, k, P, P, P, P, P, 10, 64, 0, 1e-6, q, k, dwq, dwk, work, None)  # noqa: E731
    assert call(dwq=None) == call(dwk=None) == call(work=None) == B.ERR_NULL
    assert call(work=ODD) == B.ERR_ALIGNMENT
    assert call(g=heads(h=1)) == B.ERR_INVALID_ARG
    work = L.dybit_head_norm_rope_bwd_workspace
    assert work(0, 4, 64) == 128 and work(-1, 4, 64) == 0 and work(1, 4, 0) == 0
    assert 0 < work(1, 40, 128) <= work(100000, 40, 128) == work(10 ** 9, 40, 128)


def test_append():
    call = lambda k=heads(), v=heads(), slots=P, c=cache(): B.lib().dybit_kv_append(k, v, slots, c, None)  # noqa: E731
    assert call(k=heads(n=0), v=heads(n=0)) == B.OK
    assert call(slots=None) == call(k=heads(data=None)) == call(c=cache(k_codes=None)) == call(c=cache(v_scales=None)) == B.ERR_NULL
    assert call(c=cache(k_scales=ODD)) == call(v=heads(data=0x1002)) == B.ERR_ALIGNMENT
    assert call(c=cache(kb=6)) == call(c=cache(vb=2)) == call(c=cache(kb=5)) == call(c=cache(v_signed=False)) == B.ERR_UNSUPPORTED_BITS
    assert call(v=heads(n=3)) == call(v=heads(type=1)) == call(c=cache(h=3)) == call(c=cache(d=128)) == call(c=cache(layers=2)) == B.ERR_INVALID_ARG
    for bad in (cache(page=8), cache(page=24), cache(page=2048), cache(pages=-1), cache(pages=1 << 31), cache(h=0)):
        assert call(c=bad) == B.ERR_INVALID_ARG
    assert call(k=heads(d=32), v=heads(d=32), c=cache(d=32)) == B.ERR_INVALID_ARG


def test_copy_pages():
    call = lambda c=cache(), src=P, dst=P, n=3: B.lib().dybit_kv_copy_pages(c, src, dst, n, None)  # noqa: E731
    assert call(n=0) == call(c=cache(layers=0)) == B.OK
    assert call(src=None) == call(dst=None) == call(c=cache(v_codes=None)) == B.ERR_NULL
    assert call(n=-1) == call(n=9) == call(c=cache(layers=-1)) == B.ERR_INVALID_ARG


def attention(q=None, c=None, tables=P, width=4, lengths=P, starts=None, sequences=4, most=1, longest=0, causal=1, scale=0.1, prefix=NONE, out=None,
              work=P, size=1 << 40):
    q = q or heads()
    return B.lib().dybit_kv_attention(q, c or cache(), tables, width, lengths, starts, sequences, most, longest, causal, scale, prefix, out or q, work, size, None)


def prefix(groups=1, width=4, tables=P, lengths=P, starts=P, most=4, longest=0):
    return B.KVPrefixStruct(tables, lengths, starts, groups, width, most, longest)


def test_attention():
    assert attention(q=heads(n=0)) == attention(sequences=0) == attention(most=0) == B.OK
    assert attention(tables=None) == attention(lengths=None) == B.ERR_NULL
    assert attention(q=heads(h=1)) == attention(q=heads(h=3)) == attention(q=heads(d=128)) == attention(out=heads(h=4)) == attention(out=heads(type=2)) == B.ERR_INVALID_ARG
    assert attention(width=-1) == attention(sequences=-1) == attention(most=-1) == attention(longest=-1) == attention(causal=2) == B.ERR_INVALID_ARG
    assert attention(scale=float("inf")) == attention(scale=float("nan")) == attention(sequences=1 << 16) == attention(width=1 << 31) == B.ERR_INVALID_ARG
    assert attention(c=cache(kb=6)) == B.ERR_UNSUPPORTED_BITS
    assert attention(prefix=prefix(tables=None)) == attention(prefix=prefix(lengths=None)) == attention(prefix=prefix(starts=None)) == B.ERR_NULL
    assert attention(prefix=prefix(groups=-1)) == attention(prefix=prefix(groups=5)) == attention(prefix=prefix(width=-1)) == attention(prefix=prefix(most=-1)) == B.ERR_INVALID_ARG


def test_attention_workspace():
    need = lambda q=heads(), c=cache(pages=1 << 20), width=4, n=4, most=1, longest=0, x=NONE: B.lib().dybit_kv_attention_workspace_bytes(q, c, width, n, most, longest, x)  # noqa: E731
    assert need() == 0                                    # 64 tokens are one part: nothing to join
    long = need(width=4096)
    assert long > 0 and long % (4 * 2 * 66 * 4) == 0
    assert need(width=4096, longest=64) == 0 and need(n=0) == 0 and need(q=heads(n=0)) == 0
    assert need(x=prefix()) > 0
    assert need(q=heads(h=3)) == 0                        # a call that is refused
    assert attention(c=cache(pages=1 << 20), width=4096, size=long - 1) == B.ERR_INVALID_ARG
    assert attention(c=cache(pages=1 << 20), width=4096, work=None) == B.ERR_NULL
    assert attention(c=cache(pages=1 << 20), width=4096, work=ODD) == B.ERR_ALIGNMENT


@pytest.mark.parametrize("name", ["head_norm_rope", "head_norm_rope_bwd", "kv_append", "kv_copy_pages", "kv_attention"])
def test_native_calls_check_their_argument_count(name):
    with pytest.raises(TypeError, match="arguments"):
        getattr(B._n(), name)()
