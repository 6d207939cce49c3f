"""Dense attention over packed sequences and its gradients from the definition, in float64 on the CPU, with bounds on
what a bf16 implementation may be off by.

Bounds (u = 2^-8: a value rounded to bf16 is off by at most u relative to itself).  Probabilities and dS are rounded once as
operands of the next product, results once more, everything else is fp32 (its share: F relative to the sums of magnitudes,
which covers scores of up to a few dozen with contractions over 128 channels, and sums over the lengths used here):
  out    u (sum_j P |v| + |out|)
  delta  D = dout . out is taken from rounded outputs: |dD| <= sum_c |dout_c| err(out_c)
  dv     u (sum_i P |dout| + |dv|)
  dq     u (scale sum_j |dS| |k| + |dq|) + scale sum_j P |k| |dD|
  dk     u (scale sum_i |dS| |q| + |dk|)      (D is put right before dk and dbias use it: off by F's share only)
  dbias  u |dbias|
"""
import numpy as np
import torch

U = 2.0 ** -8
F = 2e-5


def lengths_to_offsets(lengths, gap_before=0):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32) + gap_before


def visible(lq, lk, causal):
    rel = np.arange(lk)[None, :] - (np.arange(lq)[:, None] + lk - lq)
    return rel, (rel <= 0 if causal else np.ones_like(rel, dtype=bool))


def bucket_of(rel, bounds):
    return sum((rel >= b).astype(np.int64) for b in bounds) if len(bounds) else np.zeros_like(rel)


def attention(q, k, v, q_rows, k_rows, causal=False, scale=0.0, bias=None, bounds=(), dout=None):
    """q [n_q, h, d], k, v [n_k, hk, d] float64 arrays; q_rows, k_rows: (start, length) of every sequence.  Returns
    (values, errors): dicts of arrays; rows of no sequence are NaN in the values."""
    n_q, h, d = q.shape
    n_k, hk = k.shape[:2]
    sc = scale if scale > 0 else 1.0 / np.sqrt(d)
    nan = float("nan")
    val = {"out": np.full((n_q, h, d), nan), "lse": np.full((n_q, h), nan)}
    err = {"out": np.zeros((n_q, h, d)), "lse": np.zeros((n_q, h))}
    if dout is not None:
        val.update(dq=np.full((n_q, h, d), nan), dk=np.full((n_k, hk, d), nan), dv=np.full((n_k, hk, d), nan))
        err.update(dq=np.zeros((n_q, h, d)), dk=np.zeros((n_k, hk, d)), dv=np.zeros((n_k, hk, d)))
        if bias is not None:
            val["dbias"], err["dbias"] = np.zeros(bias.shape), np.zeros(bias.shape)
    for (a, lq), (b, lk) in zip(q_rows, k_rows):
        rel, seen = visible(lq, lk, causal)
        which = bucket_of(rel, bounds)
        if dout is not None:
            for x in (val, err):
                x["dk"][b:b + lk] = x["dv"][b:b + lk] = 0
        for t in range(h):
            qh, kh, vh = q[a:a + lq, t], k[b:b + lk, t // (h // hk)], v[b:b + lk, t // (h // hk)]
            s = sc * (qh @ kh.T)
            size = sc * (np.abs(qh) @ np.abs(kh).T)  # magnitudes behind a score: its fp32 error goes by them
            ok = seen
            if bias is not None:
                row = bias[t][which]
                ok = seen & (row > -1e30)
                s = s + np.where(ok, row, 0)
                size = size + np.abs(np.where(ok, row, 0))
            s = np.where(ok, s, -np.inf)
            top = np.max(s, axis=1, initial=-np.inf)
            e = np.exp(s - np.where(np.isfinite(top), top, 0)[:, None])
            total = e.sum(1)
            p = e / np.where(total > 0, total, 1)[:, None]
            with np.errstate(divide="ignore"):
                val["lse"][a:a + lq, t] = np.log(total) + np.where(np.isfinite(top), top, 0)
            f = F + 2.0 ** -21 * np.max(np.where(ok, size, 0), axis=1, initial=0)[:, None]  # of the exponentials
            err["lse"][a:a + lq, t] = f[:, 0] + 2.0 ** -22 * np.abs(np.where(total > 0, val["lse"][a:a + lq, t], 0))
            out = p @ vh
            out_err = (U + f) * (p @ np.abs(vh) + np.abs(out))
            val["out"][a:a + lq, t], err["out"][a:a + lq, t] = out, out_err
            if dout is None:
                continue
            g = dout[a:a + lq, t]
            dp = g @ vh.T
            delta = (g * out).sum(1, keepdims=True)
            d_err = (np.abs(g) * out_err).sum(1, keepdims=True) + F * (np.abs(g) * np.abs(out)).sum(1, keepdims=True)
            ds = p * (dp - delta)
            mag = p * (np.abs(g) @ np.abs(vh).T + np.abs(delta))
            ds_err, fine = p * d_err + f * mag, f * mag
            ads = np.abs(ds) + ds_err
            kv = t // (h // hk)
            val["dq"][a:a + lq, t] = sc * ds @ kh
            err["dq"][a:a + lq, t] = sc * (U * ads + ds_err) @ np.abs(kh) + U * np.abs(val["dq"][a:a + lq, t])
            val["dk"][b:b + lk, kv] += sc * ds.T @ qh
            err["dk"][b:b + lk, kv] += sc * (U * np.abs(ds) + (1 + U) * fine).T @ np.abs(qh)
            val["dv"][b:b + lk, kv] += p.T @ g
            err["dv"][b:b + lk, kv] += ((U + f) * p).T @ np.abs(g)
            if bias is not None:
                n = bias.shape[1]
                val["dbias"][t] += np.bincount(which.ravel(), ds.ravel(), minlength=n)
                err["dbias"][t] += np.bincount(which.ravel(), fine.ravel(), minlength=n)
    if dout is not None:
        for x in ("dk", "dv", "dbias"):
            if x in val:
                err[x] += U * np.abs(np.nan_to_num(val[x])) + U * err[x]
    return val, err


def check(name, got, val, err):
    """got within err of val wherever val is a number; infinities equal."""
    got, val, err = np.asarray(got, dtype=np.float64), np.asarray(val), np.asarray(err)
    where = ~np.isnan(val)
    assert not np.isnan(got[where]).any(), f"{name}: NaN at {np.argwhere(np.isnan(got) & where)[:4].tolist()}"
    inf = np.isinf(val)
    assert (got[inf] == val[inf]).all(), f"{name}: infinities differ"
    where &= ~inf
    over = np.abs(got - np.where(where, val, 0)) - (err + 1e-30)
    over = np.where(where, over, -1)
    if over.size and over.max() > 0:
        at = np.unravel_index(np.argmax(over), over.shape)
        raise AssertionError(f"{name}{at}: {got[at]} for {val[at]}, allowed {err[at]}; {int((over > 0).sum())} of {over.size} outside")


def f64(t):
    return t.detach().to(torch.float32).cpu().numpy().astype(np.float64)
