"""Dense attention: what the C boundary and the binding refuse, workspaces, bucket bounds, and the reference itself (no GPU)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import attn_ref as R
from paper_2604_05182_amd import binding as B

ADDR = 1 << 20  # stands for a device pointer: refused calls look at its alignment only


def params(n_q=100, n_k=100, n_seq=2, h_q=4, h_kv=2, d=64, bounds=None, **kw):
    p = B.lsrm_attn_params()
    p.n_q, p.n_k, p.n_seq, p.h_q, p.h_kv, p.d = n_q, n_k, n_seq, h_q, h_kv, d
    p.d_q_offsets = ADDR
    if bounds is not None:
        p._arr = (ctypes.c_int32 * max(len(bounds), 1))(*bounds)
        p.n_buckets, p.bucket_bounds = len(bounds) + 1, ctypes.cast(p._arr, ctypes.POINTER(ctypes.c_int32))
    for name, value in kw.items():
        if isinstance(value, tuple):
            getattr(p, name)[:] = value
        else:
            setattr(p, name, value)
    return p


def forward(p, q=ADDR, k=ADDR, v=ADDR, bias=None, out=ADDR, lse=None, ws=ADDR, ws_bytes=1 << 40):
    return B._lib.lsrm_attn_forward(ctypes.byref(p) if p is not None else None, q, k, v, bias, out, lse, ws, ws_bytes, None)


def backward(p, q=ADDR, k=ADDR, v=ADDR, bias=None, out=ADDR, lse=ADDR, dout=ADDR, dq=ADDR, dk=ADDR, dv=ADDR, dbias=None, ws=ADDR,
             ws_bytes=1 << 40):
    return B._lib.lsrm_attn_backward(ctypes.byref(p) if p is not None else None, q, k, v, bias, out, lse, dout, dq, dk, dv, dbias, ws,
                                     ws_bytes, None)


def bad_params():
    inv, uns = B.LSRM_ERR_INVALID_ARG, B.LSRM_ERR_UNSUPPORTED
    return [
        (params(n_q=-1, n_k=-1), inv), (params(n_seq=-1), inv), (params(h_q=0), inv), (params(h_kv=0), inv), (params(d=0), inv),
        (params(h_q=3), inv), (params(causal=2), inv), (params(scale=-1.0), inv), (params(scale=float("nan")), inv),
        (params(scale=float("inf")), inv), (params(scale=3e38), inv), (params(d_q_offsets=None), inv), (params(n_k=101), inv),
        (params(n_buckets=-1), inv), (params(n_buckets=2), inv), (params(bounds=[3, 3]), inv), (params(bounds=[3, 1]), inv),
        (params(q_stride=(4, 64)), inv), (params(k_stride=(128, 0)), inv), (params(v_stride=(-128, 64)), inv),
        (params(o_stride=((1 << 24) + 8, 64)), inv), (params(q_stride=(256, (1 << 40) + 8)), inv),
        (params(d=96), uns), (params(n_q=1 << 31, n_k=1 << 31), uns), (params(n_q=1 << 29, n_k=1 << 29, h_q=8), uns),
        (params(n_seq=1 << 24), uns), (params(bounds=list(range(64))), uns), (params(bounds=[0, (1 << 20) + 1]), uns),
        (params(bounds=[-(1 << 20) - 1]), uns), (params(bounds=[0, 1023]), uns), (params(h_q=16, h_kv=1, bounds=[0, 511], n_q=90, n_k=90), uns),
    ]


@pytest.mark.parametrize("i", range(len(bad_params())))
def test_params_are_refused(i):
    p, status = bad_params()[i]
    bias = ADDR if p.n_buckets > 0 else None
    assert forward(p, bias=bias) == status and backward(p, bias=bias) == status
    assert B.lsrm_attn_workspace_bytes(p, B.LSRM_WS_FORWARD) == B.lsrm_attn_workspace_bytes(p, B.LSRM_WS_BACKWARD) == 0


def test_pointers_are_refused():
    p, b = params(), params(bounds=[-1, 2])
    assert forward(None) == backward(None) == B.LSRM_ERR_INVALID_ARG
    for name in ("q", "k", "v", "out"):
        for value in (None, ADDR + 8):
            assert forward(p, **{name: value}) == B.LSRM_ERR_INVALID_ARG, name
    for name in ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv"):
        for value in (None, ADDR + 2):
            assert backward(p, **{name: value}) == B.LSRM_ERR_INVALID_ARG, name
    assert forward(p, lse=ADDR + 2) == B.LSRM_ERR_INVALID_ARG
    assert forward(p, bias=ADDR) == forward(b) == forward(b, bias=ADDR + 1) == B.LSRM_ERR_INVALID_ARG
    assert backward(p, bias=ADDR) == backward(b) == backward(p, dbias=ADDR) == backward(b, bias=ADDR, dbias=ADDR + 1) == B.LSRM_ERR_INVALID_ARG


def test_workspaces():
    # one query over a long cache is cut into parts; many rows need no scratch
    few = params(n_q=1, n_k=100000, n_seq=1, d_k_offsets=ADDR, causal=1)
    need = B.lsrm_attn_workspace_bytes(few, B.LSRM_WS_FORWARD)
    assert need > 0
    for ws, n in ((None, need), (ADDR + 128, need), (ADDR, need - 1), (ADDR, 0)):
        assert forward(few, ws=ws, ws_bytes=n) == B.LSRM_ERR_WORKSPACE
    assert B.lsrm_attn_workspace_bytes(params(n_q=100000, n_k=100000), B.LSRM_WS_FORWARD) == 0
    p = params()
    need = B.lsrm_attn_workspace_bytes(p, B.LSRM_WS_BACKWARD)
    assert need >= 100 * 4 * 8
    for ws, n in ((None, need), (ADDR + 64, need), (ADDR, need - 1)):
        assert backward(p, ws=ws, ws_bytes=n) == B.LSRM_ERR_WORKSPACE
    assert B.lsrm_attn_workspace_bytes(p, B.LSRM_WS_ROUTE) == 0


def test_nothing_to_do_needs_nothing():
    for p in (params(n_seq=0, d_q_offsets=None), params(n_q=0, n_k=0)):
        assert forward(p, q=None, k=None, v=None, out=None, ws=None, ws_bytes=0) == B.LSRM_OK
    assert backward(params(n_seq=0, d_q_offsets=None), q=None, k=None, v=None, out=None, lse=None, dout=None, dq=None, dk=None, dv=None,
                    ws=None, ws_bytes=0) == B.LSRM_OK


def test_the_binding_looks_at_tensors():
    q, k = torch.zeros((10, 4, 64), dtype=torch.bfloat16), torch.zeros((10, 2, 64), dtype=torch.bfloat16)
    off = torch.tensor([0, 10], dtype=torch.int32)
    for args in ((q.float(), k, k), (q, k, k[:9]), (q, k[..., :32], k[..., :32]), (q[0], k, k), (q.transpose(1, 2), k, k),
                 (q, k[:1].expand(10, 2, 64), k), (q, k, k), (q, k, k, off.long())):
        with pytest.raises(ValueError):  # (the last but one: offsets have to be on the GPU)
            B.make_attn_params(*(args if len(args) == 4 else args + (off,)))


def by_definition(n_side, max_distance, two_sided):
    """bucket of every distance by the usual rule, numbered from the farthest behind to the farthest ahead"""
    single = n_side // 2

    def side(x):
        if x < single:
            return x
        return min(n_side - 1, single + int(math.floor(math.log(x / single) / math.log(max_distance / single) * (n_side - single) + 1e-9)))

    def bucket(rel):
        if rel <= 0:
            return n_side - 1 - side(-rel)
        return n_side - 1 + (side(rel) if two_sided else 0)

    return bucket


@pytest.mark.parametrize("two_sided", [False, True])
@pytest.mark.parametrize("n_side,max_distance", [(16, 128), (32, 128), (8, 32), (4, 20), (5, 100), (2, 2), (16, 1000), (32, 4096)])
def test_bucket_bounds(n_side, max_distance, two_sided):
    bounds = B.lsrm_rel_bucket_bounds(n_side, max_distance, two_sided)
    assert len(bounds) == (2 if two_sided else 1) * (n_side - 1) and all(a < b for a, b in zip(bounds, bounds[1:]))
    bucket = by_definition(n_side, max_distance, two_sided)
    for rel in range(-max_distance - 5, max_distance + 6):
        assert sum(b <= rel for b in bounds) == bucket(rel), rel


def test_bucket_bounds_refused():
    b, n = (ctypes.c_int32 * 64)(), ctypes.c_int32()

    def call(n_side, max_distance, two_sided, bounds=b, count=ctypes.byref(n)):
        return B._lib.lsrm_rel_bucket_bounds(n_side, max_distance, two_sided, bounds, count)

    assert call(16, 128, 1) == B.LSRM_OK
    assert call(64, 4096, 0) == B.LSRM_OK and n.value == 63
    assert call(1, 128, 1) == call(16, 0, 1) == call(16, 128, 2) == call(16, 128, 1, None) == call(16, 128, 1, b, None) == B.LSRM_ERR_INVALID_ARG
    assert call(33, 128, 1) == call(65, 128, 0) == call(16, (1 << 20) + 1, 1) == call(16, 8, 1) == call(16, 10, 1) == B.LSRM_ERR_UNSUPPORTED


# ---- the reference ----------------------------------------------------------------------------------------------------
def small(seed=3, bias=True):
    rng = np.random.default_rng(seed)
    q, k, v, g = (rng.normal(size=(n, h, 8)) for n, h in ((9, 4), (11, 2), (11, 2), (9, 4)))
    return q, k, v, g, rng.normal(size=(4, 4)) if bias else None


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("biased", [False, True])
def test_reference_gradients_against_differences(causal, biased):
    q, k, v, g, bias = small(bias=biased)
    spans = [(0, 3), (4, 5)], [(0, 4), (5, 6)]
    kw = dict(causal=causal, bias=bias, bounds=(-2, 0, 1) if biased else ())
    val, _ = R.attention(q, k, v, *spans, dout=g, **kw)

    def loss(q=q, k=k, v=v, bias=bias):
        out = R.attention(q, k, v, *spans, causal=causal, bias=bias, bounds=kw["bounds"])[0]["out"]
        return np.nansum(out * g)

    h = 1e-5
    for name, x in (("q", q), ("k", k), ("v", v)) + ((("bias", bias),) if biased else ()):
        grad = np.nan_to_num(val["d" + name])
        for at in np.ndindex(*x.shape):
            if np.prod(at[:1]) % 3 == 0 or name == "bias":
                up, down = x.copy(), x.copy()
                up[at] += h
                down[at] -= h
                diff = (loss(**{name: up}) - loss(**{name: down})) / (2 * h)
                assert abs(diff - grad[at]) < 1e-7, (name, at)


def test_reference_against_the_library():
    q, k, v, _, _ = small(7)
    val, _ = R.attention(q[:, :, :], k[:9], v[:9], [(0, 9)], [(0, 9)], causal=True)
    t = [torch.from_numpy(x).transpose(0, 1)[None] for x in (q, k[:9], v[:9])]
    want = torch.nn.functional.scaled_dot_product_attention(*t, is_causal=True, enable_gqa=True)[0].transpose(0, 1).numpy()
    assert np.abs(val["out"] - want).max() < 1e-12


def test_bounds_let_rounding_pass_and_mistakes_fail():
    """a bf16 evaluation lies within the bounds; a shifted mask, a wrong bucket border or a missing scale do not"""
    rng = np.random.default_rng(1)

    def bf(x):
        return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()

    q, k, v, g = (bf(rng.normal(size=(90, 2, 32))) for _ in range(4))
    bias = bf(rng.normal(size=(2, 3)))
    span = [(0, 90)]
    kw = dict(causal=True, bias=bias, bounds=(-7, -1))
    val, err = R.attention(q, k, v, span, span, dout=g, **kw)
    rel, seen = R.visible(90, 90, True)
    which = R.bucket_of(rel, (-7, -1))
    got = {x: np.zeros_like(val[x]) for x in val}
    for h in range(2):
        s = np.where(seen, q[:, h] @ k[:, h].T / np.sqrt(32) + bias[h][which], -np.inf)
        lse = np.log(np.exp(s).sum(1))
        p = np.exp(s - lse[:, None])
        out = bf(bf(p) @ v[:, h])
        ds = p * (g[:, h] @ v[:, h].T - (g[:, h] * out).sum(1, keepdims=True))
        got["out"][:, h], got["lse"][:, h] = out, lse
        got["dq"][:, h] = bf(bf(ds) @ k[:, h] / np.sqrt(32))
        ds -= p * ds.sum(1, keepdims=True)
        got["dk"][:, h] = bf(bf(ds).T @ q[:, h] / np.sqrt(32))
        got["dv"][:, h], got["dbias"][h] = bf(bf(p).T @ g[:, h]), bf(np.bincount(which.ravel(), ds.ravel(), minlength=3))
    for name in val:
        R.check(name, got[name], val[name], err[name])
    for wrong in (dict(kw, causal=False), dict(kw, bounds=(-8, -1)), dict(kw, bounds=(-7, 0)), dict(kw, scale=0.2)):
        bad, _ = R.attention(q, k, v, span, span, dout=g, **wrong)
        for name in ("out", "dq", "dk", "dv") + (() if "scale" in wrong else ("dbias",)):  # (dbias hardly goes by the scale)
            with pytest.raises(AssertionError):
                R.check(name, bad[name], val[name], err[name])


def test_one_row_of_a_large_cache():
    """The heads of a single row may lie as far apart as the format allows: the row's own stride says nothing."""
    cache = torch.empty((8, 70000, 128), dtype=torch.bfloat16, device="meta").transpose(0, 1)
    assert B._layout("k", cache) == ((70000, 8, 128), (128, 70000 * 128))
    shape, stride = B._layout("k", cache[:1])
    assert shape == (1, 8, 128) and stride == (8 * 128, 70000 * 128)
    assert B._layout("k", cache[:, :1]) == ((70000, 1, 128), (128, 128))


@pytest.mark.parametrize("bounds, error", [([-3, 0, 1 << 32], ValueError), ([-(1 << 31) - 1, 0], ValueError), ([-3, 0.5], TypeError)])
def test_bounds_are_not_cut_to_fit(bounds, error):
    with pytest.raises(error):
        B._bounds(bounds)
    assert list(B._bounds([np.int64(-3), torch.tensor(4)])) == [-3, 4]
