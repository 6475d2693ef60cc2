"""Forms of the training operators that only the C interface has: results left out, and results at any address their type can have.
Needs an MI355X."""
import math

import numpy as np
import pytest
import torch

import train_reference as ref
from paper_2212_01185_amd import binding

pytestmark = pytest.mark.gpu

BF16, FP32 = torch.bfloat16, torch.float32
SHAPES = [(160, 128), (48, 24), (200, 264), (30, 33), (7, 13)]


def _grad(dz, x, w, off, act, dx, dw, db):
    groups, n_out, n_in = w.shape
    need = binding.load().pcc_grouped_linear_grad_workspace_bytes(x.shape[0], groups, n_in, n_out)
    space = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    at = lambda t: t.data_ptr() if t is not None else None  # noqa: E731
    rc = binding.load().pcc_grouped_linear_grad(dz.data_ptr(), dz.stride(0), x.data_ptr(), x.stride(0), w.data_ptr() if dx is not None else None,
                                                off.data_ptr(), groups, x.shape[0], n_in, n_out, binding.PCC_BF16, act, at(dx),
                                                dx.stride(0) if dx is not None else 0, at(dw), at(db), space.data_ptr() if dw is not None else None,
                                                need if dw is not None else 0, torch.cuda.current_stream().cuda_stream)
    assert rc == binding.PCC_OK


@pytest.mark.parametrize("fan_in,fan_out", SHAPES)
def test_backward_without_some_of_its_results(fan_in, fan_out):
    lengths = [300, 0, 4000, 1]
    gen = torch.Generator().manual_seed(fan_in)
    x, dz = (torch.randn(sum(lengths) + 2, n, generator=gen).to(BF16).cuda() for n in (fan_in, fan_out))
    w = (torch.randn(4, fan_out, fan_in, generator=gen) / math.sqrt(fan_in)).to(BF16).cuda()
    offsets = [0] + np.cumsum(lengths).tolist()
    off = torch.tensor(offsets).cuda()
    (dx0, dxb), (dw0, dwb), (db0, dbb) = ref.linear_grad(dz, x, w, offsets, ref.RELU)

    def fresh(*shape, dtype=FP32, shift=0):             # `shift` elements behind where vectors could be stored, 7 around it
        n = math.prod(shape)
        full = torch.full((n + 16,), 7.0, dtype=dtype, device="cuda")
        return full, full[8 + shift:8 + shift + n].view(shape)

    for with_dx, with_dw, with_db, shift in ((True, False, False, 0), (True, True, False, 0), (False, True, False, 1), (False, True, True, 1), (True, True, True, 3)):
        holders = {"dx": fresh(*x.shape, dtype=BF16, shift=2 * (shift // 2)) if with_dx else None, "dw": fresh(*w.shape, shift=shift) if with_dw else None,
                   "db": fresh(4, fan_out, shift=shift) if with_db else None}
        parts = {k: v[1] if v else None for k, v in holders.items()}
        _grad(dz, x, w, off, ref.RELU, parts["dx"], parts["dw"], parts["db"])
        for name, value, bound in (("dx", dx0, dxb), ("dw", dw0, dwb), ("db", db0, dbb)):
            if parts[name] is not None:
                ref.assert_near(parts[name], value, bound, (name, with_dx, with_dw, with_db))
                full, part = holders[name]
                first = (part.data_ptr() - full.data_ptr()) // full.element_size()
                assert (full[:first] == 7).all() and (full[first + part.numel():] == 7).all()
        if with_dx:
            assert (parts["dx"][-2:] == 7).all()


@pytest.mark.parametrize("k", [3, 5])
def test_loss_gradient_without_bits(k):
    gen = torch.Generator().manual_seed(k)
    params, rgb = torch.randn(200, 12 * k, generator=gen).cuda(), torch.randint(0, 256, (200, 3), generator=gen).to(torch.uint8).cuda()
    bits, want = binding.pcc_mixture_loss(params, rgb)
    got = torch.empty_like(want)
    stream = torch.cuda.current_stream().cuda_stream
    L = binding.load()
    assert L.pcc_mixture_loss(params.data_ptr(), 12 * k, rgb.data_ptr(), None, 200, k, 0, 1.0, None, got.data_ptr(), binding.PCC_FP32, 12 * k, stream) == binding.PCC_OK
    assert torch.equal(got, want)
    assert L.pcc_mixture_loss(params.data_ptr(), 12 * k, rgb.data_ptr(), None, 200, k, 0, 1.0, None, params.data_ptr(), binding.PCC_FP32, 12 * k, stream) == binding.PCC_OK
    assert torch.equal(params, want)                    # in place of the parameters
