"""Attention in 64 bits, sequence by sequence and head by head, and inputs for its tests."""
import numpy as np
import torch


def reference(q, k, v, q_off, k_off, causal, scale, bias=None, bucket=None, dout=None):
    """A dict of float64 arrays: out, lse, and for the bounds abs_out (sum of p |v|) and abs_s (the largest
    sum of |q| |k| scale + |bias| of a row); with dout also dq, dk, dv, dbias and their bounds' sums.
    Rows only ever meet the keys that they see."""
    f = lambda t: None if t is None else t.detach().cpu().double().numpy()  # noqa: E731
    q, k, v, bias, dout = f(q), f(k), f(v), f(bias), f(dout)
    bucket = None if bucket is None else bucket.cpu().numpy()
    (n_q, H, D), (n_k, Hk, _) = q.shape, k.shape
    r = dict(out=np.zeros_like(q), lse=np.full((n_q, H), -np.inf), abs_out=np.zeros_like(q), abs_s=np.zeros((n_q, H)))
    if dout is not None:
        for n, like in (("dq", q), ("dk", k), ("dv", v)):
            r[n], r["abs_" + n] = np.zeros_like(like), np.zeros_like(like)
        r["abs_ds"] = np.zeros((n_q, H))
        if bias is not None:
            r["dbias"], r["abs_dbias"] = np.zeros_like(bias), np.zeros_like(bias)
    q_off, k_off = q_off.cpu().numpy(), k_off.cpu().numpy()
    for s in range(len(q_off) - 1):
        q0, q1, k0, k1 = q_off[s], q_off[s + 1], k_off[s], k_off[s + 1]
        for h in range(H):
            kh = h // (H // Hk)
            for i in range(q0, q1):
                at = k1 - (q1 - i)
                last = min(k1, at + 1) if causal else k1
                if last <= k0:
                    continue
                K, V = k[k0:last, kh], v[k0:last, kh]
                z = K @ q[i, h] * scale
                size = np.abs(K) @ np.abs(q[i, h]) * scale
                if bias is not None:
                    R = len(bucket) // 2
                    b = bucket[np.clip(np.arange(k0, last) - at, -R, R) + R]
                    z = z + bias[b, h]
                    size = size + np.abs(bias[b, h])
                with np.errstate(invalid="ignore", over="ignore"):
                    top = z.max()
                    e = np.exp(z - top)
                    p = e / e.sum()
                    r["lse"][i, h] = top + np.log(e.sum())
                    r["out"][i, h] = p @ V
                r["abs_out"][i, h] = p @ np.abs(V)
                r["abs_s"][i, h] = size.max()
                if dout is None:
                    continue
                do = dout[i, h]
                dp = V @ do
                delta = p @ dp
                ds = p * (dp - delta)
                # what a gradient's rounding errors are relative to: the weight times everything that is
                # subtracted in its bracket, before anything cancels
                ads = p * (np.abs(V) @ np.abs(do) + r["abs_out"][i, h] @ np.abs(do))
                r["dv"][k0:last, kh] += p[:, None] * do
                r["abs_dv"][k0:last, kh] += p[:, None] * np.abs(do)
                r["dq"][i, h] = ds @ K * scale
                r["abs_dq"][i, h] = ads @ np.abs(K) * scale
                r["dk"][k0:last, kh] += ds[:, None] * q[i, h] * scale
                r["abs_dk"][k0:last, kh] += ads[:, None] * np.abs(q[i, h]) * scale
                if bias is not None:
                    np.add.at(r["dbias"][:, h], b, ds)
                    np.add.at(r["abs_dbias"][:, h], b, ads)
    return r


def offsets(lengths, device="cuda"):
    return torch.tensor([0, *np.cumsum(lengths)], dtype=torch.int64, device=device)


def inputs(q_lens, k_lens, heads, kv_heads, dim, dtype, seed=0, reach=0, buckets=0, causal=False, device="cuda"):
    """(q, k, v, q_off, k_off, dict of bias and bucket); k_lens None: the sequences attend to themselves."""
    from paper_2202_13538_amd import binding
    g = torch.Generator().manual_seed(seed)
    n_q, n_k = sum(q_lens), sum(q_lens if k_lens is None else k_lens)
    normal = lambda *s: torch.randn(*s, generator=g).to(dtype).to(device)  # noqa: E731
    q, k, v = normal(n_q, heads, dim), normal(n_k, kv_heads, dim), normal(n_k, kv_heads, dim)
    q_off = offsets(q_lens, device)
    k_off = q_off if k_lens is None else offsets(k_lens, device)
    how = {}
    if buckets:
        how = dict(bias=normal(buckets, heads),
                   bucket=torch.tensor(binding.distance_buckets(reach, buckets, causal), dtype=torch.int32,
                                       device=device))
    return q, k, v, q_off, k_off, how


UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16)}  # of rounding to nearest
