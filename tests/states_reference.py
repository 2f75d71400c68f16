"""The state store and its attention from their definitions, in 64 bits on the CPU (numpy), and the error that the library's arithmetic allows.

Error of an answer, derived from the number formats: with A = sum_j p_j |v_j| (p: the exact weights) per component,
  - the answer's rounding: u_out |out|, u_out = 2^-8 (bfloat16) or 2^-11 (binary16);
  - the weights' rounding to binary16: 2^-11 relative, or 2^-25 absolute where the largest weight is 1 (subnormal weights): the latter adds
    2^-25 sum_j |V_j| / sum_j (w_j / sv_j);
  - the logits, in float: their products are exact, the sum of dim terms is off by at most (dim + 8) 2^-24 sum |q_d k_d| scale, the further float
    operations (steps, logarithm, sum, exponential) by 2^-21 (|y| + 8) in units of log2; a relative error e of the weights moves the answer by at most 2 e A;
  - sums over n weights in float, in numerator and denominator: 2 n 2^-24 A.
Queries whose components lie below 2^-28 of the row's largest lose bits in binary16: 2^-39 of the row's largest per component, which the logits' term covers."""
import numpy as np
import torch


def quantise(x):
    """Codes, steps of rows [..., dim] float32, each operation one IEEE float operation as the header states it."""
    x = np.asarray(x, np.float32)
    top = np.abs(x).max(-1)
    bad = ~np.isfinite(x).all(-1)
    zero = bad | ~(top >= np.float32(2.0 ** -100))
    down = np.where(top > np.float32(2.0 ** 100), np.float32(2.0 ** -30), np.float32(1))       # exact: the product with 127 stays finite
    with np.errstate(all="ignore"):
        codes = np.rint((x * down[..., None] * np.float32(127)) / np.where(zero, np.float32(1), top * down)[..., None])
    codes = np.where(zero[..., None], 0, codes).astype(np.int8)
    step = np.where(bad, np.float32(np.nan), np.where(zero, np.float32(0), top / np.float32(127))).astype(np.float32)
    return codes, step


def store_arrays(st):
    return {n: getattr(st, n).cpu().numpy() for n in ("k_codes", "v_codes", "k_scales", "v_scales")}


def gather(a, pages, shift_page, n_pages, length):
    """(key codes, value codes [n, heads, dim], steps [n, heads] each) of the keys 0..length-1 that stand on pages of the store."""
    P = shift_page
    t = np.arange(length)
    page = pages[t // P]
    ok = (page >= 0) & (page < n_pages)
    t, page = t[ok], page[ok]
    off = t % P
    return t, (a["k_codes"][page, :, off].astype(np.float64), a["v_codes"][page, :, :, off].astype(np.float64),
               a["k_scales"][page, :, off].astype(np.float64), a["v_scales"][page, :, off].astype(np.float64))


U_OUT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def attention_rows(q, parts, scale, u_out):
    """q [T, heads, group, dim] float64; parts: list of ((kc, vc, ks, vs), seen [T, n] or None, bias).  (answers, allowed error), the same shape as q."""
    T, H, G, D = q.shape
    out, tol = np.zeros_like(q), np.zeros_like(q)
    parts = [p for p in parts if p[0][0].shape[0]]
    if not parts:
        return out, tol
    kc, vc, ks, vs = (np.concatenate([p[0][i] for p in parts]) for i in range(4))
    n = kc.shape[0]
    seen = np.concatenate([np.ones((T, p[0][0].shape[0]), bool) if p[1] is None else p[1] for p in parts], 1)
    bias = np.concatenate([np.full(p[0][0].shape[0], p[2]) for p in parts])
    with np.errstate(all="ignore"):
        for h in range(H):
            k, v = kc[:, h] * ks[:, h, None], vc[:, h] * vs[:, h, None]
            sv = np.where(vs[:, h] < 2.0 ** -100, 2.0 ** -100, vs[:, h])
            for g in range(G):
                for t in range(T):
                    m = seen[t]
                    if not m.any():
                        continue
                    z = scale * (k[m] @ q[t, h, g]) + bias[m]
                    if (z == -np.inf).all():
                        continue
                    p = np.exp(z - z.max())
                    total = p.sum()
                    out[t, h, g] = (p @ v[m]) / total
                    A = (p @ np.abs(v[m])) / total
                    y = z / np.log(2) + np.log2(sv[m])
                    w = np.exp2(y - y.max())
                    e_logit = (D + 8) * 2.0 ** -24 * abs(scale) * (np.abs(k[m]) @ np.abs(q[t, h, g])).max() + 2.0 ** -21 * (np.abs(np.where(np.isfinite(y), y, 0)).max() + np.abs(bias[m][np.isfinite(bias[m])]).max(initial=0) + 8)
                    sub = 2.0 ** -25 * np.abs(vc[m, h]).sum(0) / (w / sv[m]).sum()
                    tol[t, h, g] = u_out * np.abs(out[t, h, g]) + (2.0 ** -11 + 2 * e_logit + 2 * n * 2.0 ** -24) * A + sub + 1e-30
    return out, tol


def chunk(st, q, tables, lengths, q_start, scale):
    """(answers, allowed error) [tokens, query heads, dim] of attend_chunk; rows of tokens without a sequence are NaN."""
    a, P = store_arrays(st), st.page_size
    H, G, D = st.heads, q.shape[1] // st.heads, st.dim
    qn = q.detach().cpu().double().numpy().reshape(q.shape[0], H, G, D)
    out, tol = np.full_like(qn, np.nan), np.zeros_like(qn)
    for s in range(tables.shape[0]):
        lo, hi = int(q_start[s]), int(q_start[s + 1])
        length = min(max(int(lengths[s]), 0), tables.shape[1] * P)
        t, rows = gather(a, np.asarray(tables[s]), P, st.pages, length)
        seen = t[None, :] <= (length - (hi - lo) + np.arange(hi - lo))[:, None]
        out[lo:hi], tol[lo:hi] = attention_rows(qn[lo:hi], [(rows, seen, 0.0)], scale, U_OUT[q.dtype])
    return out.reshape(q.shape), tol.reshape(q.shape)


def passages(st, q, ids, tables, lengths, q_start, scores, weight, scale):
    a, P = store_arrays(st), st.page_size
    H, G, D = st.heads, q.shape[1] // st.heads, st.dim
    qn = q.detach().cpu().double().numpy().reshape(q.shape[0], H, G, D)
    out, tol = np.full_like(qn, np.nan), np.zeros_like(qn)
    for s in range(ids.shape[0]):
        lo, hi = int(q_start[s]), int(q_start[s + 1])
        parts = []
        for r, i in enumerate(np.asarray(ids[s])):
            if not 0 <= i < tables.shape[0]:
                continue
            b = 0.0 if scores is None else float(weight) * float(scores[s, r])
            if b == -np.inf:
                continue
            length = min(max(int(lengths[i]), 0), tables.shape[1] * P)
            _, rows = gather(a, np.asarray(tables[i]), P, st.pages, length)
            parts.append((rows, None, b))
        out[lo:hi], tol[lo:hi] = attention_rows(qn[lo:hi], parts, scale, U_OUT[q.dtype])
    return out.reshape(q.shape), tol.reshape(q.shape)


def chunk_on_gpu(st, q, tables, lengths, q_start, scale):
    """chunk() for sizes that are too many for one row at a time: the same in float64 on the GPU, a sequence and query head at a time.  Tensors."""
    H, G, D, P = st.heads, q.shape[1] // st.heads, st.dim, st.page_size
    out, tol = torch.zeros(q.shape, dtype=torch.float64, device=q.device), torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    for s in range(tables.shape[0]):
        lo, hi, n = int(q_start[s]), int(q_start[s + 1]), int(lengths[s])
        t = torch.arange(n, device=q.device)
        page, off = tables[s].long()[t // P], t % P
        seen = t[None, :] <= (n - (hi - lo) + torch.arange(hi - lo, device=q.device))[:, None]
        for h in range(H):
            ks, vs = st.k_scales[page, h, off].double(), st.v_scales[page, h, off].double()
            vc = st.v_codes[page, h, :, off].double()
            k, v = st.k_codes[page, h, off].double() * ks[:, None], vc * vs[:, None]
            for g in range(G):
                x = q[lo:hi, h * G + g].double()
                z = (scale * (x @ k.T)).masked_fill(~seen, float("-inf"))
                p = torch.softmax(z, 1)
                o, a = p @ v, p @ v.abs()
                y = z / np.log(2) + torch.log2(vs)
                w = torch.exp2(y - y.max(1, keepdim=True).values)
                e = (D + 8) * 2.0 ** -24 * abs(scale) * (x.abs() @ k.abs().T).max(1, keepdim=True).values + 2.0 ** -21 * (y.masked_fill(~seen, 0).abs().max(1, keepdim=True).values + 8)
                sub = 2.0 ** -25 * (seen.double() @ vc.abs()) / (w / vs).sum(1, keepdim=True)
                out[lo:hi, h * G + g] = o
                tol[lo:hi, h * G + g] = U_OUT[q.dtype] * o.abs() + (2.0 ** -11 + 2 * e + 2 * n * 2.0 ** -24) * a + sub + 1e-30
    return out, tol


def assert_close(got, want, tol, what=""):
    got = got.detach().cpu().double().numpy()
    assert got.shape == want.shape, what
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), f"{what}: NaN at other places"
    err = np.abs(np.where(nan, 0, got - np.where(nan, 0, want)))
    bad = err > np.where(nan, 0, tol)
    assert not bad.any(), f"{what}: off by {err[bad].max():.3g} where {np.where(nan, 0, tol)[bad].min():.3g} is allowed, at {np.argwhere(bad)[0]} of {got.shape}"
