"""Orthogonal updates with the roundings that their documentation names and no others, in torch on any device: how large an error they leave has to be
known before a kernel's can be judged.  TEST INFRASTRUCTURE ONLY."""
import torch

USUAL = (3.4445, -4.7750, 2.0315)


def significand(v, bits):
    """v (64 bits) to that many bits of significand, ties to even."""
    m, e = torch.frexp(v)
    return torch.ldexp(torch.round(torch.ldexp(m, torch.tensor(bits))), e - bits)


def pieces(v, n, bits):
    """v as n numbers of that many bits, largest first."""
    out = []
    for _ in range(n):
        out.append(significand(v, bits))
        v = v - out[-1]
    return out


def product(P, Q, fp32_sums, pairs_of):
    """P Q^T of lists of pieces: 16 columns at a time, a rounding to fp32 behind each (fp32_sums), the pieces' products that pairs_of names."""
    acc = torch.zeros(P[0].shape[0], Q[0].shape[0], dtype=torch.float64, device=P[0].device)
    K = P[0].shape[1]
    if not fp32_sums:
        return sum((P[i] @ Q[j].t().contiguous() for i, j in pairs_of), acc)
    for k in range(0, K, 16):
        for i, j in pairs_of:
            acc = (acc + P[i][:, k:k + 16] @ Q[j][:, k:k + 16].t().contiguous()).float().double()
    return acc


def orthogonalize(u, steps=5, coefs=None, eps=1e-7, operand_bits=None, n_pieces=1, fp32_sums=False, pairs_of=((0, 0),)):
    """One matrix in 64 bits; operand_bits None: nothing is rounded."""
    x = u.double()
    turned = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if turned else x
    x = x / (torch.linalg.vector_norm(x) + eps)
    cut = (lambda v: pieces(v, n_pieces, operand_bits)) if operand_bits else (lambda v: [v])
    eye = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for i in range(steps):
        a, b, c = USUAL if coefs is None else coefs[i]
        X = cut(x)
        A = cut(product(X, X, fp32_sums, pairs_of))
        B = a * eye + b * sum(A) + c * product(A, A, fp32_sums, pairs_of)
        B = cut(B.float().double() if fp32_sums else B)
        x = product(B, [p.t().contiguous() for p in X], fp32_sums, pairs_of)
    return x.t().contiguous() if turned else x


STORED = {"bf16": dict(operand_bits=11), "f32": dict(operand_bits=11, n_pieces=2, fp32_sums=True, pairs_of=((0, 0), (1, 0), (0, 1)))}


def spectrum(M, N, least, seed):
    """A matrix whose singular values run from 1 down to `least`, evenly in their logarithm."""
    g = torch.Generator().manual_seed(seed)
    S = min(M, N)
    U, V = (torch.linalg.qr(torch.randn(n, S, generator=g, dtype=torch.float64))[0] for n in (M, N))
    return (U * torch.logspace(0, torch.log10(torch.tensor(least)).item(), S, dtype=torch.float64)) @ V.t()
