"""The attention sublayer's entry points refuse what they cannot take before they touch the device; the bucket rule, in whole numbers."""
import ctypes as C

import pytest

from paper_2601_12917_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(B.LIB_PATH):
        from paper_2601_12917_amd.build import build
        build()
    return B.lib()


def _heads(data=0x1000, batch=64, token=64, head=64):
    return B.zgr_heads(data, batch, token, head)


def _attention(**kw):
    base = dict(dtype=B.ZGR_BF16, batch=2, n_q=8, n_k=8, n_head=2, n_kv_head=2, head_dim=64, causal=0, scale=0.1)
    base.update(kw)
    return B.zgr_attention(**base)


def _message():
    return B.lib().zgr_last_error(None).decode()


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), B.ZGR_ERR_DTYPE), (dict(batch=-1), B.ZGR_ERR_SHAPE), (dict(n_q=-1), B.ZGR_ERR_SHAPE), (dict(n_k=(1 << 26) + 1), B.ZGR_ERR_SHAPE), (dict(n_head=0), B.ZGR_ERR_SHAPE),
    (dict(n_head=3), B.ZGR_ERR_SHAPE), (dict(n_kv_head=0), B.ZGR_ERR_SHAPE), (dict(head_dim=4), B.ZGR_ERR_SHAPE), (dict(head_dim=136), B.ZGR_ERR_SHAPE), (dict(head_dim=20), B.ZGR_ERR_SHAPE),
    (dict(causal=2), B.ZGR_ERR_CONFIG), (dict(scale=0.0), B.ZGR_ERR_CONFIG), (dict(scale=-1.0), B.ZGR_ERR_CONFIG), (dict(scale=float("nan")), B.ZGR_ERR_CONFIG),
    (dict(scale=float("inf")), B.ZGR_ERR_CONFIG), (dict(bias=0x2000), B.ZGR_ERR_NULL), (dict(bias=0x2000, bias_map=0x3000), B.ZGR_ERR_SHAPE),
    (dict(bias=0x2000, bias_map=0x3000, bias_buckets=4, bias_reach=1025), B.ZGR_ERR_SHAPE), (dict(bias=0x2000, bias_map=0x3000, bias_buckets=4, bias_reach=-1), B.ZGR_ERR_SHAPE),
    (dict(bias=0x2001, bias_map=0x3000, bias_buckets=4, bias_reach=1), B.ZGR_ERR_SHAPE), (dict(k_lengths=0x3002), B.ZGR_ERR_SHAPE),
    (dict(batch=1 << 20, n_q=1 << 26, n_head=2), B.ZGR_ERR_SHAPE)])
def test_attention_descriptions_are_refused(lib, kw, status):
    how, h = _attention(**kw), _heads()
    assert lib.zgr_attention_forward(C.byref(how), h, h, h, h, 0x1000, 0x1000, 1 << 30, None) == status, _message()
    assert lib.zgr_attention_backward(C.byref(how), h, h, h, h, h, 0x1000, h, h, h, None, 0x1000, 1 << 30, None) == status, _message()
    assert lib.zgr_attention_workspace(C.byref(how)) == 0 and lib.zgr_attention_backward_workspace(C.byref(how)) == 0


def test_attention_pointers_and_workspaces_are_refused(lib):
    how, h = _attention(), _heads()
    f = lambda q=h, k=h, v=h, o=h, lse=0x1000, ws=0x1000, n=1 << 30: lib.zgr_attention_forward(C.byref(how), q, k, v, o, lse, ws, n, None)
    assert lib.zgr_attention_forward(None, h, h, h, h, 0x1000, 0x1000, 1 << 30, None) == B.ZGR_ERR_NULL
    assert f(q=None) == f(k=_heads(None)) == f(v=None) == f(o=None) == f(lse=None) == B.ZGR_ERR_NULL
    assert f(q=_heads(0x1008)) == f(k=_heads(token=65)) == f(v=_heads(head=4)) == f(o=_heads(batch=63)) == f(lse=0x1002) == B.ZGR_ERR_SHAPE
    if lib.zgr_attention_workspace(C.byref(how)):
        assert f(ws=None) == B.ZGR_ERR_NULL and f(ws=0x1010) == f(n=8) == B.ZGR_ERR_WORKSPACE
    one = _attention(batch=1, n_head=1, n_kv_head=1, n_q=0)                  # nothing to do, whatever the pointers
    assert lib.zgr_attention_forward(C.byref(one), None, None, None, None, None, None, 0, None) == B.ZGR_OK
    b = lambda dout=h, lse=0x1000, dq=h, dk=h, db=None, ws=0x1000, n=1 << 30: lib.zgr_attention_backward(C.byref(how), dout, h, h, h, h, lse, dq, dk, h, db, ws, n, None)
    assert b(dout=None) == b(lse=None) == b(dq=None) == b(dk=_heads(0)) == b(ws=None) == B.ZGR_ERR_NULL
    assert b(dout=_heads(token=1)) == b(dq=_heads(0x1004)) == b(db=0x1001) == B.ZGR_ERR_SHAPE
    assert b(ws=0x1010) == b(n=lib.zgr_attention_backward_workspace(C.byref(how)) - 1) == B.ZGR_ERR_WORKSPACE and "needed" in _message()


def _rotation(**kw):
    base = dict(dtype=B.ZGR_BF16, rows=4, q_heads=2, k_heads=1, head_dim=64, rot_dim=32, interleaved=0, n_positions=10, eps=1e-6, table=0x1000, positions=0x1000)
    base.update(kw)
    return B.zgr_rotation(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), B.ZGR_ERR_DTYPE), (dict(rows=-1), B.ZGR_ERR_SHAPE), (dict(q_heads=0, k_heads=0), B.ZGR_ERR_SHAPE), (dict(q_heads=-1), B.ZGR_ERR_SHAPE), (dict(head_dim=0), B.ZGR_ERR_SHAPE),
    (dict(head_dim=12), B.ZGR_ERR_SHAPE), (dict(head_dim=264), B.ZGR_ERR_SHAPE), (dict(rot_dim=4), B.ZGR_ERR_SHAPE), (dict(rot_dim=72), B.ZGR_ERR_SHAPE), (dict(eps=-1.0), B.ZGR_ERR_CONFIG),
    (dict(eps=float("nan")), B.ZGR_ERR_CONFIG), (dict(interleaved=2), B.ZGR_ERR_CONFIG), (dict(n_positions=0), B.ZGR_ERR_SHAPE), (dict(table=None), B.ZGR_ERR_NULL), (dict(positions=None), B.ZGR_ERR_NULL),
    (dict(positions=0x1002), B.ZGR_ERR_SHAPE), (dict(q_gain=0x1001), B.ZGR_ERR_SHAPE), (dict(rows=(1 << 31) - 1, q_heads=65536), B.ZGR_ERR_SHAPE)])
def test_rotations_are_refused(lib, kw, status):
    how, h = _rotation(**kw), _heads()
    assert lib.zgr_norm_rotate(C.byref(how), h, h, h, h, None) == status, _message()
    assert lib.zgr_norm_rotate_backward(C.byref(how), h, h, h, h, h, h, 0x1000, 0x1000, 1 << 30, None) == status, _message()


def test_rotation_pointers_and_workspaces_are_refused(lib):
    how, h = _rotation(), _heads()
    assert lib.zgr_norm_rotate(None, h, h, h, h, None) == B.ZGR_ERR_NULL and lib.zgr_norm_rotate_backward_workspace(None) == 0
    assert lib.zgr_norm_rotate(C.byref(how), None, h, h, h, None) == lib.zgr_norm_rotate(C.byref(how), h, h, h, _heads(None), None) == B.ZGR_ERR_NULL
    assert lib.zgr_norm_rotate(C.byref(how), h, _heads(0x1008), h, h, None) == lib.zgr_norm_rotate(C.byref(how), h, h, _heads(token=33), h, None) == B.ZGR_ERR_SHAPE
    n = lib.zgr_norm_rotate_backward_workspace(C.byref(how))
    back = lambda dg=0x1000, ws=0x1000, n=n: lib.zgr_norm_rotate_backward(C.byref(how), h, h, h, h, h, h, dg, ws, n, None)
    assert back(ws=None) == B.ZGR_ERR_NULL and back(n=n - 1) == back(ws=0x1010) == B.ZGR_ERR_WORKSPACE and back(dg=0x1002) == B.ZGR_ERR_SHAPE


def test_dropout_is_refused(lib):
    def f(rows=4, cols=8, xt=0, x=0x1000, st=0, res=None, out=0x1000, p=0.1, step=0, first=0):
        return lib.zgr_dropout_add(rows, cols, xt, x, cols, None, st, res, cols, out, cols, p, 1, step, 0, first, None)
    assert f(xt=2) == f(st=-1) == B.ZGR_ERR_DTYPE
    assert f(rows=-1) == f(cols=0) == f(rows=(1 << 31) - 1, cols=(1 << 31) - 1) == B.ZGR_ERR_SHAPE
    assert f(p=-0.1) == f(p=1.0) == f(p=float("nan")) == f(p=1 - 2.0 ** -34) == f(step=1 << 32) == f(first=1 << 32) == B.ZGR_ERR_CONFIG
    assert f(x=None) == f(out=None) == B.ZGR_ERR_NULL
    assert f(x=0x1001) == f(out=0x1002) == f(res=0x1002) == B.ZGR_ERR_SHAPE
    assert f(rows=0, x=None, out=None) == B.ZGR_OK

    def b(rows=4, cols=8, st=0, dout=0x1000, xt=0, dx=0x1000, db=0x1000, p=0.1, ws=0x1000, n=1 << 20):
        return lib.zgr_dropout_add_backward(rows, cols, st, dout, cols, xt, dx, cols, db, p, 1, 0, 0, 0, ws, n, None)
    assert b(st=3) == B.ZGR_ERR_DTYPE and b(p=1.0) == B.ZGR_ERR_CONFIG and b(dout=None) == b(dx=None) == b(ws=None) == B.ZGR_ERR_NULL
    assert b(ws=0x1020) == b(n=16) == B.ZGR_ERR_WORKSPACE and b(db=0x1002) == B.ZGR_ERR_SHAPE
    assert lib.zgr_dropout_add_backward_workspace(-1, 4) == 0 and lib.zgr_dropout_add_backward_workspace(4, 0) == 0


def test_bucket_rule_in_whole_numbers(lib):
    """Bucket exact + m holds the distances a with (a / exact)^(n - exact) in [(reach / exact)^m, (reach / exact)^(m + 1))."""
    for buckets in (1, 2, 3, 4, 8, 16, 31, 32, 33, 64, 100):
        for reach in (0, 1, 2, 7, 8, 16, 31, 64, 100, 128, 333, 512, 1024):
            for causal in (0, 1):
                if not causal and buckets < 2:
                    continue
                out = (C.c_int32 * (2 * reach + 1))()
                assert lib.zgr_relative_buckets(buckets, reach, causal, out) == B.ZGR_OK
                n = buckets if causal else buckets // 2
                exact = max(1, n // 2)
                for d in range(-reach, reach + 1):
                    a = max(0, -d) if causal else abs(d)
                    got = out[d + reach] - (n if d > 0 and not causal else 0)
                    assert 0 <= got < n
                    if a < exact or reach <= exact:
                        assert got == min(a, n - 1)
                    else:
                        m = got - exact
                        power = lambda m: (a ** (n - exact) * exact ** m >= reach ** m * exact ** (n - exact))
                        assert (got == n - 1 or not power(m + 1)) and (m <= 0 or power(m)), (buckets, reach, causal, d, got)
    assert lib.zgr_relative_buckets(4, 8, 0, None) == B.ZGR_ERR_NULL
    assert lib.zgr_relative_buckets(1, 8, 0, out) == lib.zgr_relative_buckets(4, 1025, 0, out) == lib.zgr_relative_buckets(4, -1, 0, out) == B.ZGR_ERR_SHAPE
    assert lib.zgr_relative_buckets(4, 8, 2, out) == B.ZGR_ERR_CONFIG


def test_python_refuses_what_the_library_cannot_see():
    torch = pytest.importorskip("torch")
    from paper_2601_12917_amd import sublayer as S
    x = torch.zeros(2, 4, 2, 32)
    with pytest.raises(ValueError):
        S.attention(x, x, x)                                                 # not on the GPU
    with pytest.raises(TypeError):
        S.attention(x.half(), x.half(), x.half())
    with pytest.raises(ValueError):
        S.attention(x, x[:1], x[:1])
    with pytest.raises(ValueError):
        S.attention(x, x, x, bias=torch.zeros(4, 3), bias_map=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError):
        S.attention(x, x, x, k_lengths=torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        S.norm_rotate(None, None, None, None, None, None)
    with pytest.raises(ValueError):
        S.norm_rotate(x[0], x[0, :1], None, None, None, None)
