"""Norm per head and rotation in 64 bits on the CPU, and their gradients, from the formulas (test infrastructure)."""
import torch


def axis_of_pair(sections, dealt):
    if not dealt:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    left, out, a = list(sections), [], 0
    while sum(left):
        if left[a]:
            left[a] -= 1
            out.append(a)
        a = (a + 1) % len(left)
    return out


def rotation(positions, inv_freq, sections, dealt, rotary, d, adjacent):
    """[T, d, d] matrices R with y = R n for each token: orthogonal, so that the gradient turns by the transpose."""
    T = positions.shape[-1]
    R = torch.eye(d, dtype=torch.float64).repeat(T, 1, 1)
    if rotary == 0:
        return R
    pos = positions.reshape(-1, T).double()
    for i, a in enumerate(axis_of_pair(sections, dealt)):
        t = pos[a] * inv_freq[i].double()
        x, y = (2 * i, 2 * i + 1) if adjacent else (i, i + rotary // 2)
        R[:, x, x] = R[:, y, y] = torch.cos(t)
        R[:, x, y], R[:, y, x] = -torch.sin(t), torch.sin(t)
    return R


def forward(x, w, R, norm, eps):
    """x [T, H, d] any type -> [T, H, d] in 64 bits."""
    n = x.double()
    if norm:
        n = n / torch.sqrt((n * n).mean(-1, keepdim=True) + eps)
        if w is not None:
            n = n * w.double()
    return torch.einsum("tij,thj->thi", R, n)


def backward(x, w, R, norm, eps, dy):
    """(dx, dw or None) in 64 bits, by the formulas."""
    g = torch.einsum("tji,thj->thi", R, dy.double())
    if not norm:
        return g, None
    x = x.double()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    dw = (g * x * r).sum((0, 1))
    h = g * w.double() if w is not None else g
    return r * (h - x * r * r * (h * x).mean(-1, keepdim=True)), dw
