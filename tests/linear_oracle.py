"""Linear attention with a decay for each head, token by token in 64-bit torch: the definition, and what bounds the kernels' roundings."""
import torch

BF16_STEP, F32_STEP = 2.0 ** -8, 2.0 ** -24     # half a step, relative to the value


def sequences(B, T, cu):
    return [(b * T, (b + 1) * T) for b in range(B)] if cu is None else [(int(x), int(y)) for x, y in zip(cu[:-1], cu[1:])]


def _flat(x):
    return x.double().reshape((-1,) + x.shape[2:])


def forward(Q, K, V, log_decay, scale, S0, cu):
    """O [B,T,H,d_v], S [sequences,H,d_k,d_v]."""
    B, T = Q.shape[:2]
    seqs, lam = sequences(B, T, cu), torch.exp(log_decay.double())[:, None, None]
    q, k, v = _flat(Q), _flat(K), _flat(V)
    out, S = torch.zeros_like(v), torch.zeros(len(seqs), Q.shape[2], Q.shape[3], V.shape[3], dtype=torch.float64, device=Q.device)
    if S0 is not None:
        S += S0.double()
    for s, (beg, end) in enumerate(seqs):
        for t in range(beg, end):
            S[s] = lam * S[s] + k[t][:, :, None] * v[t][:, None, :]
            out[t] = scale * torch.einsum("hk,hkv->hv", q[t], S[s])
    return out.reshape(V.shape), S


def backward(dO, Q, K, V, log_decay, scale, S0, dS, cu):
    """dQ, dK, dV, dS0 by the recurrence's own derivative."""
    B, T = Q.shape[:2]
    seqs, lam = sequences(B, T, cu), torch.exp(log_decay.double())[:, None, None]
    q, k, v, x = _flat(Q), _flat(K), _flat(V), _flat(dO)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    shape = (len(seqs), Q.shape[2], Q.shape[3], V.shape[3])
    S = torch.zeros(shape, dtype=torch.float64, device=Q.device) + (0 if S0 is None else S0.double())
    G = torch.zeros(shape, dtype=torch.float64, device=Q.device) + (0 if dS is None else dS.double())
    for s, (beg, end) in enumerate(seqs):
        for t in range(beg, end):
            S[s] = lam * S[s] + k[t][:, :, None] * v[t][:, None, :]
            dq[t] = scale * torch.einsum("hkv,hv->hk", S[s], x[t])
        for t in range(end - 1, beg - 1, -1):
            G[s] += scale * q[t][:, :, None] * x[t][:, None, :]
            dk[t] = torch.einsum("hkv,hv->hk", G[s], v[t])
            dv[t] = torch.einsum("hkv,hk->hv", G[s], k[t])
            G[s] *= lam
    return dq.reshape(Q.shape), dk.reshape(K.shape), dv.reshape(V.shape), G


def within(got, ref, absolute, bf16_terms, out_bf16, depth):
    """Whether every element is inside its bound.  ``absolute``: the same sums with every term's absolute value, which no sum of rounded terms can leave by more than
    the roundings' shares of it: ``bf16_terms`` roundings to bf16 of operands that are themselves computed (P or the state: each term meets one), the
    output's own rounding, and fp32 roundings, ``depth`` of them on a term's way (products, sums and the factors' exponentials)."""
    bound = absolute * (bf16_terms * BF16_STEP + depth * F32_STEP) * 1.01
    if out_bf16:
        bound = bound + BF16_STEP * (ref.abs() + bound)
    diff = (got.double() - ref).abs()
    bad = ~(diff <= bound + 1e-30)
    assert not bool(bad.any()), "worst %.3g of its bound, %d of %d outside" % (float((diff / (bound + 1e-30)).nan_to_num(float("inf")).max()), int(bad.sum()), bad.numel())
