"""What attention, its key ranges and dropout refuse, through the C ABI and through the torch layers: every refusal
comes before anything touches a device, so this runs without one."""
import ctypes as C
import math

import pytest
import torch

from paper_2606_30634_amd import attention, binding as B, dropout

P, Q, R = 1 << 20, 1 << 40, 1 << 41  # aligned addresses, far from each other, that are never read


def _refused(fn, *args):
    with pytest.raises(B.StageError) as e:
        fn(*args)
    assert e.value.code == B.STAGE_EINVAL and B.last_error()


S3 = B._STRIDES
PARAMS = dict(batch=2, queries=5, keys=9, heads=4, kv_heads=2, hd=64, bf=1, qs=(1280, 256, 64), ks=(1152, 128, 64),
              vs=(1152, 128, 64), start=None, end=None, first=None, slopes=None, scale=0.125, cap=0.0)


def _params(**kw):
    d = dict(PARAMS, **kw)
    for n in ("qs", "ks", "vs"):
        d[n] = S3(*d[n])
    return B.AttentionParams(*d.values())


BAD_PARAMS = [dict(batch=-1), dict(batch=(1 << 24) + 1), dict(queries=-1), dict(queries=(1 << 30) + 1), dict(keys=-2),
              dict(keys=(1 << 30) + 1), dict(heads=3), dict(heads=0, kv_heads=0), dict(kv_heads=0), dict(heads=8192, kv_heads=1),
              dict(hd=48), dict(hd=256), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan),
              dict(cap=-1.0), dict(cap=math.inf), dict(cap=math.nan), dict(cap=1e-44), dict(cap=2.0 ** -61), dict(cap=2.0 ** 101), dict(scale=2.0 ** -61), dict(scale=2.0 ** 61), dict(scale=2.0 ** -60, cap=2.0 ** 90), dict(start=P), dict(end=P),
              dict(start=P, end=P + 2), dict(first=P + 1), dict(slopes=P + 2), dict(qs=(1280, 256, 60)), dict(ks=(1152, -128, 64)),
              dict(vs=(1152, 128, 4)), dict(qs=(1 << 41, 256, 64)), dict(ks=(1152, (1 << 24) + 8, 64)),
              dict(batch=1 << 20, queries=1 << 20)]
FWD = dict(q=P, k=P, v=P, o=Q, o32=None, lse=R, ws=1 << 42, nb=1 << 40, stream=None)


@pytest.mark.parametrize("bad", BAD_PARAMS)
def test_params_refused(bad):
    _refused(B.attention_forward, _params(**bad), *FWD.values())
    g = _grads()
    _refused(B.attention_backward, _params(**bad), P, P, P, P, P, P, g, 1 << 42, 1 << 40, None)


@pytest.mark.parametrize("bad", [dict(q=None), dict(k=None), dict(v=None), dict(q=P + 8), dict(v=P + 4), dict(o=None), dict(o=Q + 2),
                                 dict(lse=None), dict(lse=R + 2), dict(o=P + 16), dict(o32=P), dict(o32=Q), dict(lse=Q),
                                 dict(o32=Q + (1 << 30) + 4)])
def test_forward_refuses(bad):
    _refused(B.attention_forward, _params(), *dict(FWD, **bad).values())


def test_forward_refuses_o_f32_of_fp32_and_small_workspaces():
    wide = dict(qs=(1280, 256, 64), bf=0)
    _refused(B.attention_forward, _params(**wide), *dict(FWD, o32=Q + (1 << 30)).values())
    long = _params(batch=1, queries=1, keys=32768)
    need = B.attention_workspace_bytes(long)
    assert need > 0
    for ws, nb in ((None, need), (1 << 42, need - 1), ((1 << 42) + 128, need)):
        _refused(B.attention_forward, long, *dict(FWD, ws=ws, nb=nb).values())


def _grads(**kw):
    d = dict(os=(1280, 256, 64), dos=(1280, 256, 64), dqs=(1280, 256, 64), dks=(1152, 128, 64), dvs=(1152, 128, 64), dq=Q, dk=R, dv=R + (1 << 30), wide=0)
    d.update(kw)
    for n in ("os", "dos", "dqs", "dks", "dvs"):
        d[n] = S3(*d[n])
    return B.AttentionGrads(*d.values())


BWD = dict(q=P, k=P, v=P, o=P, lse=P, dout=P, g=None, ws=1 << 42, nb=1 << 40, stream=None)


@pytest.mark.parametrize("bad", [dict(q=None), dict(o=None), dict(lse=None), dict(lse=P + 2), dict(dout=None), dict(dout=P + 8),
                                 dict(ws=None), dict(nb=64), dict(ws=(1 << 42) + 16), dict(o=P + 8), dict(g=dict(os=(1280, 252, 64))), dict(g=dict(os=(1280, 2, 64), wide=1)),
                                 dict(g=dict(dq=None)), dict(g=dict(dk=None)), dict(g=dict(dv=R + 4)), dict(g=dict(dq=P)),
                                 dict(g=dict(dk=P + 256)), dict(g=dict(dk=Q)), dict(g=dict(dv=R)), dict(g=dict(dv=R + 128)),
                                 dict(g=dict(dqs=(1280, 0, 64))), dict(g=dict(dks=(1152, 64, 64))), dict(g=dict(dvs=(0, 128, 64))),
                                 dict(g=dict(dks=(1152, 128, 4))), dict(g=dict(dos=(1280, 256, -64))),
                                 # heads of one packed row that meet: k's end where v's begin + 32
                                 dict(g=dict(dq=Q, dk=Q + 512, dv=Q + 704, dqs=(2560, 512, 64), dks=(2560, 512, 64), dvs=(2560, 512, 64))),
                                 dict(g=dict(dq=Q, dk=Q + 512, dv=Q + 960, dqs=(2560, 512, 64), dks=(2560, 512, 64), dvs=(2560, 512, 64)))])
def test_backward_refuses(bad):
    g = _grads(**bad.get("g", {}))
    a = dict(BWD, **dict(bad, g=g))
    _refused(B.attention_backward, _params(), *a.values())


def test_null_structs():
    null = C.POINTER(B.AttentionParams)()
    assert B.LIB.attention_forward(null, *FWD.values()) == B.STAGE_EINVAL
    assert B.LIB.attention_workspace_bytes(null) == 0 and B.LIB.attention_backward_workspace_bytes(null) == 0
    a = dict(BWD, g=C.POINTER(B.AttentionGrads)())
    assert B.LIB.attention_backward(C.byref(_params()), *a.values()) == B.STAGE_EINVAL


def test_nothing_to_do():
    B.attention_forward(_params(batch=0), None, None, None, None, None, None, None, 0, None)
    B.attention_forward(_params(queries=0), None, P, P, None, None, None, None, 0, None)
    B.attention_key_ranges(0, 5, None, None, None, None, None)
    B.attention_key_ranges(5, 0, None, None, None, None, None)
    B.dropout_add(0, 7, None, 7, None, 0, None, 7, 0, 0.5, 0, 0, None)


RNG = dict(batch=2, length=100, ids=P, flags=P, start=Q, end=R, stream=None)


@pytest.mark.parametrize("bad", [dict(batch=-1), dict(length=-1), dict(length=(1 << 30) + 1), dict(batch=(1 << 24) + 1),
                                 dict(batch=1 << 20, length=1 << 23), dict(ids=None), dict(start=None), dict(end=None),
                                 dict(ids=P + 2), dict(start=Q + 1), dict(end=R + 2), dict(start=P), dict(end=P + 64), dict(end=Q + 64)])
def test_key_ranges_refuse(bad):
    _refused(B.attention_key_ranges, *dict(RNG, **bad).values())


DROP = dict(rows=4, cols=100, x=P, ldx=100, r=P, ldr=100, out=Q, ldo=100, bf=0, p=0.5, seed=1, offset=2, stream=None)


@pytest.mark.parametrize("bad", [dict(rows=-1), dict(cols=-1), dict(rows=1 << 30, cols=1 << 30), dict(p=-0.1), dict(p=1.0),
                                 dict(p=math.nan), dict(p=65535.5 / 65536), dict(ldx=99), dict(ldr=99), dict(ldo=99), dict(x=None),
                                 dict(out=None), dict(x=P + 2), dict(r=P + 1), dict(out=Q + 2), dict(out=P + 16), dict(out=P, ldo=101),
                                 dict(out=P + 400, r=P + 800), dict(bf=1, x=P + 1), dict(ldx=(1 << 40) + 1)])
def test_dropout_refuses(bad):
    _refused(B.dropout_add, *dict(DROP, **bad).values())


@pytest.mark.parametrize("call", [
    lambda z: attention.key_ranges(z(2, 8).int()),                                # not on a GPU
    lambda z: attention.key_ranges(None),
    lambda z: attention.key_ranges(z(8).int()),
    lambda z: attention.attention(z(1, 2, 2, 64), z(1, 4, 2, 64), z(1, 4, 2, 64)),
    lambda z: attention.attention(None, z(1, 4, 2, 64), z(1, 4, 2, 64)),
    lambda z: attention.attention(z(2, 2, 64), z(1, 4, 2, 64), z(1, 4, 2, 64)),
    lambda z: attention.attention(z(1, 2, 2, 64).double(), z(1, 4, 2, 64), z(1, 4, 2, 64)),
    lambda z: attention.attention_backward(z(1, 2, 2, 64), z(1, 4, 2, 64), z(1, 4, 2, 64), attention.Attention(), z(1, 2, 2, 64)),
    lambda z: dropout.dropout_add(z(4, 8), z(4, 8), 0.1, 1),
    lambda z: dropout.dropout_add(z(4, 8), None, 0.1, 1),
    lambda z: dropout.dropout_backward(None, 0.1, 1),
    lambda z: dropout.dropout_backward(z(8), 0.1, 1)])
def test_torch_layers_refuse(call):
    with pytest.raises(ValueError):
        call(lambda *s: torch.zeros(*s))
