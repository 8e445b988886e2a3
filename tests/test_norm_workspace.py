"""The workspace of a group norm: a call takes what its own plan wants and more, and refuses less before it has written anything."""
import ctypes as C

import pytest
import torch

import paper_2202_02365_b200 as mg
from paper_2202_02365_b200 import api

pytestmark = pytest.mark.gpu


class Call:
    """mg_group_norm_backward of equal samples with a workspace of any size."""

    def __init__(self, ctx, samples, per, channels, groups, dtype, shift=0):
        g = torch.Generator("cuda").manual_seed(1)
        n = samples * per * channels
        self.ctx, self.channels = ctx, channels
        self.x, self.d_y = (torch.randn(n + shift, generator=g, device="cuda").to(dtype)[shift:].view(samples * per, channels) for _ in range(2))
        self.mean, self.rstd = torch.zeros((samples, groups), device="cuda"), torch.ones((samples, groups), device="cuda")
        self.spec = api.NormSpec(samples * per, channels, groups, api.ROW_TYPES[dtype], 0, 1.0, 0, None, per, None, None, None)
        need = C.c_size_t(0)
        ctx._check(ctx.lib.mg_group_norm_workspace(ctx.handle, C.byref(self.spec), 1, C.byref(need)))
        self.need = need.value
        self.work = torch.empty(self.need, dtype=torch.uint8, device="cuda")

    def run(self, size):
        out, d_w, d_b = torch.zeros_like(self.x), torch.zeros(self.channels, device="cuda"), torch.zeros(self.channels, device="cuda")
        c = self.channels
        rc = self.ctx.lib.mg_group_norm_backward(self.ctx.handle, C.byref(self.spec), self.x.data_ptr(), c, self.d_y.data_ptr(), c, self.mean.data_ptr(), self.rstd.data_ptr(),
                                                 out.data_ptr(), c, d_w.data_ptr(), d_b.data_ptr(), self.work.data_ptr() if size else None, size,
                                                 torch._C._cuda_getCurrentRawStream(0))
        torch.cuda.synchronize()
        return rc, (out, d_w, d_b)


# Rows of single elements, in 40 tiles of 16 runs of channels, want a third of what the same rows aligned do, in 240 tiles of two
@pytest.mark.parametrize("samples,per,channels,groups,dtype,shift,less", [(40, 300, 4096, 32, torch.float16, 0, False), (40, 300, 4096, 32, torch.float16, 1, True), (2000, 1, 1020, 4, torch.float32, 1, False), (3, 5000, 96, 3, torch.bfloat16, 0, False),
                                                                          (100, 30, 602, 2, torch.float32, 0, False)])
def test_the_least_that_a_call_takes(samples, per, channels, groups, dtype, shift, less):
    call = Call(mg.Context(0), samples, per, channels, groups, dtype, shift)
    rc, want = call.run(call.need)
    assert rc == 0 and want[0].any()
    refused, taken = 0, call.need
    rc, out = call.run(refused)
    assert rc == -5 and not any(t.any() for t in out)
    while taken - refused > 32:
        at = (refused + taken) // 32 * 16
        rc, out = call.run(at)
        if rc == 0:
            taken = at
            assert all(torch.equal(a, b) for a, b in zip(out, want))
        else:
            refused = at
            assert rc == -5 and not any(t.any() for t in out)
    assert taken < call.need or not less
