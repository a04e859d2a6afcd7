"""CPU checks of the attention operators: their argument errors (no kernel is launched by these
calls), empty calls, workspace sizes, and the binding's refusals."""
import ctypes

import pytest
import torch

from paper_2609_33496_amd import cham
from paper_2609_33496_amd.attention_block import AttentionBlock

NAN, INF = float("nan"), float("inf")
BIG = 1 << 31


def _heads(**kw):
    d = dict(p=64, token=256, head=64, H=4, type=2)
    d.update(kw)
    return cham._Heads(*[d[k] for k, _ in cham._Heads._fields_])


def _rotate(**kw):
    d = dict(T=3, D=64, R=64, layout=0, norm=1, eps=1e-6, amp=1.0, qg=64, kg=64, qg_type=0, kg_type=1, pos=64, freq=64)
    d.update(kw)
    return cham._Rotate(*[d[k] for k, _ in cham._Rotate._fields_])


def _cache(**kw):
    d = dict(pages=8, H=4, D=64, page=16, type=3, k=64, v=64, ks=64, vs=64)
    d.update(kw)
    return cham._Cache(*[d[k] for k, _ in cham._Cache._fields_])


def _attn(**kw):
    d = dict(B=1, T=3, D=64, causal=1, scale=0.125, pad=0, cu_q=None, q=_heads(), o=_heads(p=4096))
    d.update(kw)
    return cham._Attn(*[d[k] for k, _ in cham._Attn._fields_])


BAD_HEADS = [
    (dict(p=None), cham.EINVAL), (dict(p=72), cham.EINVAL), (dict(token=60), cham.EINVAL), (dict(token=260), cham.EINVAL),
    (dict(head=56), cham.EINVAL), (dict(head=68), cham.EINVAL), (dict(H=-1), cham.EINVAL), (dict(H=65537), cham.ESHAPE),
    (dict(type=3), cham.EFORMAT), (dict(type=-1), cham.EFORMAT),
]
BAD_ROTATE = [
    (dict(T=-1), cham.EINVAL), (dict(T=BIG), cham.ESHAPE), (dict(D=0), cham.EINVAL), (dict(D=60, R=0), cham.ESHAPE),
    (dict(D=136), cham.ESHAPE), (dict(R=-2), cham.EINVAL), (dict(R=7), cham.EINVAL), (dict(R=66), cham.EINVAL),
    (dict(layout=2), cham.EFORMAT), (dict(norm=2), cham.EINVAL), (dict(eps=-1.0), cham.EINVAL), (dict(eps=NAN), cham.EINVAL),
    (dict(eps=INF), cham.EINVAL), (dict(amp=NAN), cham.EINVAL), (dict(amp=INF), cham.EINVAL), (dict(qg=72), cham.EINVAL),
    (dict(kg_type=3), cham.EFORMAT), (dict(pos=None), cham.EINVAL), (dict(pos=66), cham.EINVAL), (dict(freq=None), cham.EINVAL),
    (dict(freq=68), cham.EINVAL),
]
BAD_CACHE = [
    (dict(pages=0), cham.EINVAL), (dict(pages=1 << 27), cham.ESHAPE), (dict(H=0), cham.EINVAL), (dict(page=8), cham.ESHAPE),
    (dict(page=48), cham.ESHAPE), (dict(page=65536), cham.ESHAPE), (dict(D=72), cham.ESHAPE), (dict(D=144), cham.ESHAPE),
    (dict(type=0), cham.EFORMAT), (dict(type=4), cham.EFORMAT), (dict(k=None), cham.EINVAL), (dict(v=72), cham.EINVAL),
    (dict(ks=None), cham.EINVAL), (dict(vs=66), cham.EINVAL), (dict(type=2), cham.EINVAL),  # scales beside 16 bits
]


@pytest.mark.parametrize("kw,status", BAD_ROTATE)
def test_rotate_refusals(kw, status):
    L, h = cham.lib(), _heads()
    assert L.cham_norm_rotate(_rotate(**kw), h, h, h, h, None) == status
    assert L.cham_cache_write(_cache(), 64, _rotate(**kw), h, h, h, h, None) == status


@pytest.mark.parametrize("kw,status", BAD_HEADS)
def test_heads_refusals(kw, status):
    L, h, bad = cham.lib(), _heads(), _heads(**kw)
    for at in range(4):
        args = [bad if i == at else h for i in range(4)]
        assert L.cham_norm_rotate(_rotate(), *args, None) in (status, cham.EINVAL, cham.EFORMAT)
    assert L.cham_norm_rotate(_rotate(), bad, bad, h, h, None) in (status, cham.EFORMAT)
    for args in ((bad, bad, h, h), (h, h, bad, bad)):
        assert L.cham_cache_write(_cache(), 64, _rotate(), *args, None) in (status, cham.EINVAL, cham.EFORMAT)
    assert L.cham_cache_read(_cache(), 64, 2, 64, 1, 3, bad, bad, None) in (status, cham.EINVAL)
    assert L.cham_attention(_attn(), bad, bad, 3, None, 256, 1 << 40, None) in (status, cham.EINVAL, cham.EFORMAT)
    assert L.cham_attention(_attn(q=bad, o=bad), h, h, 3, None, 256, 1 << 40, None) in (status, cham.EINVAL)
    assert L.cham_attention_workspace_bytes(_attn(q=bad, o=bad), 4) == 0


@pytest.mark.parametrize("kw,status", BAD_CACHE)
def test_cache_refusals(kw, status):
    L, h, c = cham.lib(), _heads(), _cache(**kw)
    assert L.cham_cache_write(c, 64, _rotate(), h, h, h, h, None) == status
    assert L.cham_cache_read(c, 64, 2, 64, 1, 3, h, h, None) == status
    assert L.cham_cache_attention(_attn(), c, 64, 2, 64, 256, 1 << 40, None) == status


def test_other_refusals():
    L, h, r, c = cham.lib(), _heads(), _rotate(), _cache()
    assert L.cham_norm_rotate(None, h, h, h, h, None) == cham.EINVAL
    assert L.cham_norm_rotate(r, h, None, h, h, None) == cham.EINVAL
    assert L.cham_norm_rotate(r, h, _heads(H=2), h, h, None) == cham.EINVAL
    assert L.cham_norm_rotate(r, h, _heads(type=1), h, h, None) == cham.EFORMAT
    assert L.cham_norm_rotate(r, h, _heads(token=512), h, h, None) == cham.EINVAL  # in place with other strides
    assert L.cham_cache_write(c, None, r, h, h, h, h, None) == cham.EINVAL
    assert L.cham_cache_write(c, 66, r, h, h, h, h, None) == cham.EINVAL
    assert L.cham_cache_write(c, 64, r, h, None, None, None, None) == cham.EINVAL
    assert L.cham_cache_write(c, 64, r, h, h, h, None, None) == cham.EINVAL
    assert L.cham_cache_write(c, 64, r, _heads(H=2), h, None, None, None) == cham.EINVAL
    assert L.cham_cache_write(c, 64, _rotate(D=32, R=32), h, h, None, None, None) == cham.EINVAL
    assert L.cham_cache_write(c, 64, r, h, _heads(type=1), None, None, None) == cham.EFORMAT
    assert L.cham_cache_read(c, None, 2, 64, 1, 3, h, h, None) == cham.EINVAL
    assert L.cham_cache_read(c, 64, 2, None, 1, 3, h, h, None) == cham.EINVAL
    assert L.cham_cache_read(c, 64, -1, 64, 1, 3, h, h, None) == cham.EINVAL
    assert L.cham_cache_read(c, 64, 2, 64, 1, 3, h, _heads(type=0), None) == cham.EFORMAT
    assert L.cham_cache_read(c, 64, 2, 64, 1 << 24, 3, h, h, None) == cham.ESHAPE
    assert L.cham_cache_read(c, 64, BIG, 64, 1, 3, h, h, None) == cham.ESHAPE


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), cham.EINVAL), (dict(B=1 << 24), cham.ESHAPE), (dict(T=-1), cham.EINVAL), (dict(T=BIG), cham.ESHAPE), (dict(D=60), cham.ESHAPE),
    (dict(D=136), cham.ESHAPE), (dict(B=2), cham.EINVAL), (dict(B=0), cham.EINVAL), (dict(causal=2), cham.EINVAL), (dict(scale=0.0), cham.EINVAL),
    (dict(scale=-1.0), cham.EINVAL), (dict(scale=NAN), cham.EINVAL), (dict(scale=INF), cham.EINVAL), (dict(cu_q=66), cham.EINVAL),
    (dict(q=_heads(type=0), o=_heads(type=0)), cham.EFORMAT), (dict(o=_heads(type=1)), cham.EFORMAT), (dict(q=_heads(H=6), o=_heads(H=6)), cham.EINVAL),
    (dict(o=_heads(H=8)), cham.EINVAL), (dict(T=1 << 29, q=_heads(H=16), o=_heads(H=16)), cham.ESHAPE),
])
def test_attention_refusals(kw, status):
    L, h, a = cham.lib(), _heads(), _attn(**kw)
    assert L.cham_attention(a, h, h, a.T if a.T > 0 else 3, None, 256, 1 << 40, None) == status
    assert L.cham_cache_attention(a, _cache(), 64, 2, 64, 256, 1 << 40, None) == status
    assert L.cham_attention_workspace_bytes(a, 4) == 0


def test_attention_other_refusals():
    L, h, a = cham.lib(), _heads(), _attn()
    need = L.cham_attention_workspace_bytes(a, 4)
    assert need > 0
    assert L.cham_attention(None, h, h, 3, None, 256, need, None) == cham.EINVAL
    assert L.cham_attention(a, h, None, 3, None, 256, need, None) == cham.EINVAL
    assert L.cham_attention(a, h, _heads(H=2), 3, None, 256, need, None) == cham.EINVAL
    assert L.cham_attention(a, h, _heads(type=1), 3, None, 256, need, None) == cham.EFORMAT
    assert L.cham_attention(a, h, h, -1, None, 256, need, None) == cham.EINVAL
    assert L.cham_attention(_attn(B=3), h, h, 4, None, 256, need, None) == cham.EINVAL  # keys of 4 / 3 rows
    assert L.cham_attention(a, h, h, 3, 66, 256, need, None) == cham.EINVAL
    assert L.cham_attention(a, _heads(token=1 << 24), h, 3, None, 256, need, None) == cham.ESHAPE
    assert L.cham_attention(a, h, h, 1000, None, None, need, None) == cham.EWORKSPACE
    assert L.cham_attention(a, h, h, 1000, None, 320, need, None) == cham.EWORKSPACE
    assert L.cham_attention(_attn(T=1), h, h, 1000, None, 256, 0, None) == cham.EWORKSPACE
    assert L.cham_attention(_attn(o=_heads()), h, h, 3, None, 256, need, None) == cham.EINVAL  # over its queries
    c = _cache()
    assert L.cham_cache_attention(a, c, None, 2, 64, 256, need, None) == cham.EINVAL
    assert L.cham_cache_attention(a, c, 64, 2, None, 256, need, None) == cham.EINVAL
    assert L.cham_cache_attention(a, c, 64, -1, 64, 256, need, None) == cham.EINVAL
    assert L.cham_cache_attention(a, c, 64, BIG, 64, 256, need, None) == cham.ESHAPE
    assert L.cham_cache_attention(a, _cache(D=32), 64, 2, 64, 256, need, None) == cham.EINVAL
    assert L.cham_cache_attention(a, _cache(type=1, ks=None, vs=None), 64, 2, 64, 256, need, None) == cham.EFORMAT
    assert L.cham_cache_attention(a, c, 64, 200, 64, 256, 1024, None) == cham.EWORKSPACE


def test_empty_calls():
    L, none = cham.lib(), _heads(p=None)
    r = _rotate(T=0, pos=None, freq=None)
    assert L.cham_norm_rotate(r, none, none, none, none, None) == cham.OK
    assert L.cham_norm_rotate(_rotate(), *[_heads(p=None, H=0)] * 4, None) == cham.OK
    assert L.cham_cache_write(_cache(), None, r, none, none, none, none, None) == cham.OK
    assert L.cham_cache_read(_cache(), None, 0, None, 0, 0, none, none, None) == cham.OK
    assert L.cham_attention(_attn(B=0, T=0, q=none, o=none), none, none, 0, None, None, 0, None) == cham.OK
    assert L.cham_cache_attention(_attn(B=0, T=0, q=none, o=none), _cache(), None, 0, None, None, 0, None) == cham.OK


def test_binding_refuses_host_tensors_and_wrong_shapes():
    q = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        cham.norm_rotate(q, q)
    with pytest.raises(ValueError):
        cham.norm_rotate(None, None)
    with pytest.raises(ValueError):
        cham.norm_rotate(q[0], None)
    with pytest.raises(ValueError):
        cham.attention(q, q, q)
    with pytest.raises(ValueError):
        cham.attention(q, q, q, batch=3)
    with pytest.raises(ValueError):
        cham.attention(q, q, q, cu_k=torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        cham.attention(q, q, q, batch=1, cu_q=torch.zeros(2, dtype=torch.int32))
    k = torch.zeros(2, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        cham.Cache(k, k)  # on the host
    with pytest.raises(ValueError):
        cham.Cache(k, k.half())
    with pytest.raises(ValueError):
        cham.Cache(k.float(), k.float())
    with pytest.raises(ValueError):
        cham.Cache(k[0], k[0])


def test_attention_block_refuses_weights_that_do_not_fit():
    w = torch.zeros(64, 128)
    with pytest.raises(ValueError):
        AttentionBlock(torch.zeros(3 * 128, 64), w, heads=3)
    with pytest.raises(ValueError):
        AttentionBlock(torch.zeros(3 * 128 - 1, 64), w, heads=2)
    with pytest.raises(ValueError):
        AttentionBlock(torch.zeros(3 * 128, 64), w, heads=2, q_weight=torch.ones(64))


def test_structures_have_the_headers_sizes():
    assert ctypes.sizeof(cham._Heads) == 32 and ctypes.sizeof(cham._Rotate) == 72
    assert ctypes.sizeof(cham._Cache) == 56 and ctypes.sizeof(cham._Attn) == 104
