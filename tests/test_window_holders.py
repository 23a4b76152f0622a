"""What Rope and Heads refuse when they are made: tensors whose type or order the kernels would misread, and more pairs than there are frequencies (no GPU)."""
import dataclasses

import pytest
import torch

import paper_2605_19218_amd as rk


class OnDevice:
    """A tensor as the holders look at it, said to be on a device."""
    is_cuda = True

    def __init__(self, t):
        self.t, self.dtype, self.shape = t, t.dtype, t.shape

    def __getattr__(self, name):
        return getattr(self.t, name)


def positions(*shape, dtype=torch.int32):
    return torch.zeros(*shape, dtype=dtype)


def frequencies(n=8, dtype=torch.float32):
    return torch.ones(n, dtype=dtype)


@pytest.mark.parametrize("wrap", [lambda t: t, OnDevice])
def test_rope(wrap):
    make = lambda pos=positions(3, 2, 6), inv=frequencies(), **m: rk.Rope(wrap(pos), wrap(inv), **m)
    r = make()
    assert r.strides == (12, 6) and r.n_axes == 3 and r.axis == bytes(8)
    assert make(axis=[0, 1, 2]).c().n_pairs == 3                     # the first of inv_freq
    assert make(pos=positions(3, 2, 9)[:, :, :6]).strides == (18, 9)
    assert make(pos=positions(2, 6, 3).permute(2, 0, 1)[:, :, :1]).strides == (1, 18)      # one token: nothing steps along tokens
    for dtype in (torch.int64, torch.int16, torch.float32, torch.uint8):
        with pytest.raises(ValueError, match="pos"):
            make(pos=positions(3, 2, 6, dtype=dtype))
    for dtype in (torch.float64, torch.bfloat16, torch.float16):
        with pytest.raises(ValueError, match="inv_freq"):
            make(inv=frequencies(dtype=dtype))
    with pytest.raises(ValueError, match="pos"):
        make(pos=positions(2, 6, 3).permute(2, 0, 1))                # axes last in memory
    with pytest.raises(ValueError, match="pos"):
        make(pos=positions(3, 2, 12)[:, :, ::2])
    with pytest.raises(ValueError, match="pos"):
        make(pos=positions(2, 6))
    with pytest.raises(ValueError, match="inv_freq"):
        make(inv=frequencies(16)[::2])
    with pytest.raises(ValueError, match="pos"):
        dataclasses.replace(r, pos=wrap(positions(3, 2, 6, dtype=torch.int64)), strides=None, n_axes=None)


def test_more_pairs_than_frequencies():
    pos, inv = OnDevice(positions(3, 2, 6)), OnDevice(frequencies(8))
    assert rk.Rope(pos, inv, axis=[1] * 8).c().n_pairs == 8
    for axis in ([0] * 9, bytes(64)):
        with pytest.raises(ValueError, match="axis"):
            rk.Rope(pos, inv, axis=axis)
    with pytest.raises(ValueError, match="axis"):
        dataclasses.replace(rk.Rope(pos, inv), inv_freq=OnDevice(frequencies(7)))


def test_heads():
    x = torch.zeros(2, 4, 7, 128)
    assert rk.Heads(x).strides == (3584, 896, 128)
    assert rk.Heads(x.transpose(1, 2)).strides == (3584, 128, 896)
    assert rk.Heads(x[:1].expand(2, 4, 7, 128)).strides == (0, 896, 128)
    for bad in (x.transpose(2, 3), torch.zeros(2, 4, 7, 256)[..., ::2], x[..., :1].expand(2, 4, 7, 128)):
        with pytest.raises(ValueError, match="channels"):
            rk.Heads(bad)
    assert rk.Heads(x.transpose(2, 3), strides=(8, 8, 8)).strides == (8, 8, 8)       # (given: the data is an address)
    assert rk.Heads(4096, strides=(8, 8, 8)).strides == (8, 8, 8)
