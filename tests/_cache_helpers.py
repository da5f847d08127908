"""Inputs and tolerances shared by the tests of the paged cache.

Tolerances, h the half step of the type (2^-8 bf16, 2^-24 fp32), e = 2^-24.

Rotation: x cos - y sin with one product rounded and one fused add is off by
at most e |y sin| + e |result| <= 2 e (|x| + |y|), then h of the result.

Attention: a score is a sum of D products; scale log2(e) is rounded once and
multiplies it: off by at most (D + 3) e reach, reach = scale sum |q||k| (the
multiplication by log2(e) cancels against the exponential's ln 2).  The exponent's
difference to the maximum adds e of itself, at most 2 e reach.  exp2 is good to one unit in
the last place, 2 e.  So a probability before normalisation is off by
r = (D + 5) e reach + 2 e of itself.  Sums over n keys, in whatever order and with the
rescaling of each part (an exponential and a product each, at most one for 32 keys),
add at most (n + 3 n / 32 + 8) e.  Numerator and denominator have that error
each.  With bf16 values the numerator's probabilities are rounded once more (h).  All of it
is relative to sum p |v|; the result's own rounding is h |out|.
"""
import numpy as np

E = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": E}


def torch_dtype(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def f64(t):
    return t.detach().double().cpu().numpy()


def dev(a, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def trees(g, B, N):
    """Parents: any node before."""
    return np.stack([[0] + [int(g.integers(0, n)) for n in range(1, N)] for _ in range(B)]).astype(np.int32)


class Cache:
    """A pool of pages in a random order, its table, and contexts of the given
    lengths that it has room for (with N more tokens)."""

    def __init__(self, g, lens, N, H, D, S, dtype, layers=None, spare=2, shared=False):
        import torch
        self.S, self.lens = S, np.array(lens, np.int32)
        need = max(1, -(-(int(max(lens)) + N) // S))
        B = len(lens)
        pages = B * need + spare
        order = g.permutation(pages)[:B * need].astype(np.int32).reshape(B, need)
        used = -(-(np.maximum(self.lens, 0).astype(np.int64) + N) // S)
        self.table = np.where(np.arange(need) < used[:, None], order, -1).astype(np.int32)
        lead = () if layers is None else (layers,)
        dt = torch_dtype(dtype)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(int(g.integers(1 << 30)))
        if shared:  # keys and values of a page side by side
            both = torch.randn(*lead, pages, 2, H, S, D, generator=gen, device="cuda").to(dt)
            self.k, self.v = both[..., 0, :, :, :], both[..., 1, :, :, :]
        else:
            self.k, self.v = (torch.randn(*lead, pages, H, S, D, generator=gen, device="cuda").to(dt) for _ in range(2))
        self.d_table, self.d_lens = dev(self.table), dev(self.lens)

    def row(self, b, j):
        return int(self.table[b, j // self.S]), j % self.S


def attention_tolerance(out, mass, reach, n, D, dtype):
    h = HALF[dtype]
    r = (D + 5) * E * reach[..., None] + 2 * E + (n + 3 * n / 32 + 8) * E
    return (2 * r + (h if dtype == "bf16" else 0.0)) * mass * 1.01 + h * np.abs(out)


def check_attention(got, want, mass, reach, n, dtype, label=""):
    g = f64(got)
    assert g.shape == want.shape
    assert np.array_equal(np.isnan(g), np.isnan(want)), f"{label}: NaN in other places"
    tol = attention_tolerance(want, mass, reach, n, want.shape[-1], dtype)
    fine = np.isfinite(want) & np.isfinite(tol)
    assert np.array_equal(g[~np.isfinite(want) & ~np.isnan(want)], want[~np.isfinite(want) & ~np.isnan(want)]), label
    over = np.where(fine, np.abs(g - np.where(fine, want, 0.0)) - np.where(fine, tol, 0.0), -1.0)
    assert (over <= 0).all(), (f"{label}: off by {np.abs(g - want).flat[over.argmax()]} at "
                               f"{np.unravel_index(over.argmax(), over.shape)}, {want.flat[over.argmax()]} wanted")
