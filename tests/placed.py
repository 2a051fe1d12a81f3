"""Tensors of a call in the layouts that callers have: contiguous, column blocks at an odd offset of wider rows ("odd"), the batch outermost ("batch"); what
surrounds an output is watched.  And comparisons with values in 64 bits."""
import numpy as np
import torch

DEV = "cuda:0"
NAN = float("nan")
TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16}


def up(a, dtype=torch.float32):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def down(t):
    return None if t is None else t.double().cpu().numpy()


def room(n):
    """A workspace whose old contents are NaNs as floats."""
    return torch.full((max(int(n), 1),), 0xFF, dtype=torch.uint8, device=DEV)


class Placed:
    def __init__(self, seed, layout="plain"):
        self.rng, self.layout, self.outer = np.random.default_rng(seed), layout, []

    def place(self, t):
        if self.layout == "plain" or t is None:
            return t
        if t.dim() == 3 and self.layout == "batch":
            return t.transpose(0, 1).contiguous().transpose(0, 1)
        wide = torch.full((*t.shape[:-1], t.shape[-1] + 5), NAN, dtype=t.dtype, device=DEV)
        view = wide[..., 3:3 + t.shape[-1]]
        view.copy_(t)
        self.outer.append(wide)
        return view

    def normal(self, shape, s=1.0, dtype=torch.float32):
        return self.place(up(self.rng.standard_normal(shape) * s, dtype))

    def empty(self, shape, dtype=torch.float32):
        return self.place(torch.full(shape, NAN, dtype=dtype, device=DEV))

    def clean(self):
        """Whether everything around the tensors is as it was."""
        return all(bool(torch.cat([w[..., :3], w[..., -2:]], -1).isnan().all()) for w in self.outer)


def near(got, want, what="", norm_of=None, bits=17):
    """32-bit values: 2^-bits of the norm and 8 times that of the largest one; bf16 one rounding more, 2^-9 of the value itself, of which twice is
    allowed.  norm_of: what the values are sums of, where they cancel."""
    wide = got.dtype == torch.float32
    g, w = got.detach().double().cpu().numpy(), np.asarray(want, np.float64)
    assert g.shape == w.shape, what
    assert np.isfinite(g).all(), what
    if not w.size:
        return
    base = np.abs(w if norm_of is None else norm_of)
    err, top, norm, small = np.abs(g - w), base.max(), np.linalg.norm(base), 2.0 ** -bits
    assert np.linalg.norm(err) <= small * norm + (0.0 if wide else 2.0 ** -8 * np.linalg.norm(w)) + 1e-30, (what, np.linalg.norm(err) / max(norm, 1e-300))
    assert (err <= 8 * small * top + (0.0 if wide else 2.0 ** -8 * np.abs(w)) + 1e-30).all(), (what, (err / max(top, 1e-300)).max())
