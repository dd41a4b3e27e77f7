"""The 8-bit norm's stream: what it adds and leaves."""
import numpy as np
import pytest

from oracle import model_ops_ref as ref
from tests.test_gpu_model_ops import U, check, host, margins, placed, torch_and_ops
from tests.test_gpu_rms_norm import BF16, F32, SHAPES, data, rsqrt_bound

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,dim,ld,shift", SHAPES)
@pytest.mark.parametrize("x_type,s_type", [(BF16, F32), (BF16, BF16), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("in_place", [False, True])
def test_8bit_norm_of_a_stream(tokens, dim, ld, shift, x_type, s_type, in_place):
    torch, ops = torch_and_ops()
    dt = lambda name: getattr(torch, name)
    x, s = data(11, tokens, dim, x_type), data(12, tokens, dim, s_type, 3.0)
    gain = 1 + torch.randn(dim, generator=torch.Generator().manual_seed(3)) * 0.2
    X, S = placed(x, dt(x_type), ld, shift), placed(s, dt(s_type), ld, shift)
    ho, ok = (S, lambda: True) if in_place else margins(tokens, dim, dt(s_type), ld, shift)
    out, scales, h = ops.rms_norm_8bit(X, gain.cuda(), residual=S, eps=1e-5, residual_out=ho)
    assert h is ho and ok()
    want = (torch.as_tensor(x).float() + torch.as_tensor(s).float()).to(dt(s_type))     # one rounding, and the type's
    assert torch.equal(h.cpu(), want)
    y = ref.rms_norm(want.double().numpy(), gain.double().numpy(), 1e-5)
    rel = rsqrt_bound(dim) + 3 * U
    want_scales = ref.e4m3_scales(y)
    check(scales, want_scales, want_scales * (rel + 2 * U), "scales")
    each = np.repeat(host(scales), 128, axis=1)[:, :dim]
    # half a step of 3 bits of mantissa, or of the least code (2^-9 of the scale)
    bound = np.maximum(np.abs(y) * 2.0 ** -4, each * 2.0 ** -10) * (1 + 4 * rel) + np.abs(y) * (rel + 3 * U)
    check(torch.as_tensor(host(out.float()) * each), y, bound, "values")
