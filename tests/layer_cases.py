"""Coded layers for the tests: codes, codebook and scales drawn from a seed, and the layer's weights in float64."""
import numpy as np
import torch

from oracle import idkm_oracle as orc

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {t: torch.finfo(t).eps / 2 for t in DTYPES.values()}


class Layer:
    def __init__(self, rows, cols, k, d, group, dtype, seed=0):
        rng = np.random.default_rng([seed, rows, cols, k, d])
        self.rows, self.cols, self.k, self.d, self.group, self.dtype = rows, cols, k, d, group, dtype
        self.codes = rng.integers(0, k, size=rows * cols // d)
        self.C = torch.from_numpy(rng.standard_normal((k, d)).astype(np.float32)).to(dtype)
        self.S = None
        if group:
            self.S = torch.from_numpy(np.exp(rng.standard_normal((rows, -(-cols // group)))).astype(np.float32))
        self.words = torch.from_numpy(orc.pack_codes(self.codes, k).view(np.int32))

    def unscaled(self):
        return self.C.double()[torch.from_numpy(self.codes)].reshape(self.rows, self.cols)

    def scales(self):
        if self.S is None:
            return torch.ones(self.rows, self.cols, dtype=torch.float64)
        return self.S.double().repeat_interleave(min(self.group, self.cols), 1)[:, : self.cols]

    def weights(self):
        return self.unscaled() * self.scales()

    def on_gpu(self, binding):
        return binding.CodesLayer(self.words.cuda(), self.rows, self.cols, self.C.cuda(), None if self.S is None else self.S.cuda(),
                                  self.group)

    def rounds_weights(self):
        """Whether a product that writes the layer out rounds its weights to the type."""
        return self.S is not None and self.dtype != torch.float32


def draw(shape, dtype, seed):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32)).to(dtype)


def sum_error(terms, length):
    """Bound of a float32 sum's error: every one of `length` additions is off by at most half a step of a partial sum, which is
    at most the sum of the terms' sizes; signs are independent, so the errors add up like a walk (four deviations), plus one
    rounding of each product and scale."""
    return (4 * length ** 0.5 + 4) * 2.0 ** -24 * terms


def check(got, ref, bound, what=""):
    got = got.detach().double().cpu()
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    off = (got - ref).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), float((off / bound.clamp(min=1e-300))[bad].max()),
                                 [tuple(x) for x in bad.nonzero()[:4].tolist()])
