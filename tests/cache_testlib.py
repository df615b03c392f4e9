"""Plain implementations, in 64 bits, of the operators around the paged cache, and the inputs of their tests."""
import numpy as np
import torch

from paper_2602_05305_amd import flashblock as fb

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}      # a rounding's largest relative error


def axis_of_pair(axis_pairs):
    return np.repeat(np.arange(len(axis_pairs)), axis_pairs)


def angles(positions, inv_freq, axis_pairs):
    """positions int [.., n_axes] -> [.., pairs], in extended precision, reduced to a turn."""
    a = positions[..., axis_of_pair(axis_pairs)].astype(np.longdouble) * inv_freq.astype(np.longdouble)
    two_pi = 2 * np.arctan2(np.longdouble(0), np.longdouble(-1))
    return np.asarray(a - two_pi * np.rint(a / two_pi), dtype=np.float64)


def members(pairs, layout):
    j = np.arange(pairs)
    return (j, j + pairs) if layout == fb.FB_ROTARY_HALVES else (2 * j, 2 * j + 1)


def rotate(x, angle, layout, inverse=False):
    """x [B, heads, n, d] float64, angle [B, n, pairs]: the rows turned."""
    x, y = x.copy(), x
    a, b = members(angle.shape[-1], layout)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None] * (-1 if inverse else 1)
    x[..., a], x[..., b] = y[..., a] * c - y[..., b] * s, y[..., a] * s + y[..., b] * c
    return x


def rotate_bound(x, positions, inv_freq, axis_pairs, layout, dtype, want):
    """What the fp32 arithmetic and the final rounding can be off by.  Relative to |x| + |y| of a pair: the fraction of a turn rounded to
    32 bits (pi 2^-25), sine and cosine (2 steps, 2^-23), two products and a sum (3 x 2^-24); the turns, three roundings of 2^-53."""
    a, b = members(sum(axis_pairs), layout)
    size = np.zeros_like(x)
    size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    far = np.zeros(positions.shape[:-1] + x.shape[-1:])
    far[..., a] = far[..., b] = np.abs(positions[..., axis_of_pair(axis_pairs)].astype(np.float64)) * inv_freq    # (|-2^31| is no int32)
    unit = np.pi * 2.0 ** -25 + 2.0 ** -23 + 3 * 2.0 ** -24 + 3 * 2.0 ** -53 * far[:, None]
    moved = np.ones(x.shape[-1], dtype=bool)
    moved[np.concatenate([a, b])] = False
    err = size * unit
    return np.where(moved, 0.0, HALF_STEP[dtype] * (np.abs(want) + err) + err)


def inv_freq(pairs, theta=10000.0):
    return (theta ** (-np.arange(pairs) / pairs)).astype(np.float32)


def rows_tensor(rng, dtype, B, heads, n, d, token_major):
    """[B, heads, n, d], dense or as a view of a token-major buffer with other columns on both sides."""
    x = torch.from_numpy(rng.standard_normal((B, heads, n, d)).astype(np.float32)).to(DEV).to(TORCH[dtype])
    if not token_major:
        return x.contiguous()
    buf = torch.randn(B, n, heads + 3, d, device=DEV).to(TORCH[dtype])
    view = buf[:, :, 1:1 + heads].transpose(1, 2)
    view.copy_(x)
    return view


def f64(t):
    return t.detach().double().cpu().numpy()


def check(got, want, bound, what):
    err = np.abs(f64(got) - want)
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, worst {np.max(np.where(bad, err - bound, 0)):.3e} over {np.max(bound):.3e}"
