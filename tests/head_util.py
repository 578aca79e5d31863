"""Buffers and bounds of the head's GPU tests."""
import numpy as np
import torch

from paper_1910_00932_amd import binding as B

TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
CDT = {"f32": B.TSM_F32, "bf16": B.TSM_BF16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}     # one rounding to the type, relative to the value
U = 2.0 ** -24                                    # one rounding in fp32


class Guarded:
    """An output of `shape` filled with NaN, with 64 elements of a pattern in front and behind that nothing may touch."""

    def __init__(self, shape, dtype):
        n = int(np.prod(shape))
        self.n = n
        self.all = torch.full((n + 128,), 7.5, dtype=dtype, device="cuda")
        self.t = self.all[64:64 + n].view(*shape)
        self.t.fill_(float("nan"))

    def np(self):
        assert bool((self.all[:64] == 7.5).all()) and bool((self.all[64 + self.n:] == 7.5).all()), "written outside"
        return self.t.double().cpu().numpy()


def values(shape, seed, dtype, scale=1.0, shift=0.0):
    """Normal values as both sides see them: on the GPU in the storage type, and in 64 bits."""
    rng = np.random.default_rng(seed)
    t = torch.from_numpy((rng.standard_normal(shape) * scale + shift).astype(np.float32)).to(TDT[dtype])
    return t.cuda(), t.double().numpy()


def scratch(nbytes):
    """A workspace of exactly the bytes asked for, full of NaN patterns."""
    return torch.full((nbytes,), 255, dtype=torch.uint8, device="cuda") if nbytes else None


def within(got, want, bound, what):
    """Element by element; NaN and infinities have to agree."""
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), (what, "NaN at other places")
    rest = ~fine & ~np.isnan(want)
    assert np.array_equal(got[rest], want[rest]), (what, "infinities at other places")
    off = np.abs(got - want)[fine]
    room = np.broadcast_to(bound, want.shape)[fine]
    bad = off > room
    assert not bad.any(), (what, int(bad.sum()), "of", bad.size, "outside; worst ratio", float((off / np.maximum(room, 1e-300)).max()))
