"""Values of the serving operators where a tolerance would hide a fault: codes exactly as defined, every bit of f32 entries, the ends of the range."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2208_10391_b200 as mom
from oracle import serving as ref
from test_gpu_serving import TYPES, dense, host, pack, ptr, stream, weights

pytestmark = pytest.mark.gpu

KIND = {v[0]: v[1] for v in TYPES.values()}


# ---- norm

def norm(x, weight, out, group=0, eps=1e-5):
    rows, cols = x.shape
    y = torch.empty(rows, cols, dtype=TYPES[out][0], device="cuda")
    s = torch.full((rows, ref.groups_of(cols, group)), float("nan"), device="cuda") if out in ("e4m3", "int8") else None
    d = mom.mom_rms_norm_desc(rows, cols, KIND[x.dtype], TYPES[out][1], KIND[weight.dtype], group, eps)
    mom.mom_rms_norm(d, ptr(x), None, None, ptr(weight), ptr(y), ptr(s), stream())
    torch.cuda.synchronize()
    return y, s


def check_codes(x, weight, out, group, eps=1e-5):
    """Scales and codes from the call's own y in f32: s = max |y| / Q (0 below 2^-100), codes y / s to nearest, each operation rounded to f32 once.  Equal, not close."""
    y, _ = norm(x, weight, "f32", 0, eps)
    q, s = norm(x, weight, out, group, eps)
    rows, cols = x.shape
    g = group or cols
    n = ref.groups_of(cols, group)
    v = torch.nn.functional.pad(y, (0, n * g - cols)).view(rows, n, g)
    m = v.abs().amax(2)                                      # (hands NaN on)
    top = torch.tensor(ref.TOP[out], device="cuda")
    want_s = torch.where(m < 2.0 ** -100, torch.zeros_like(m), m / top)
    v = torch.where(want_s[..., None] == 0, torch.zeros_like(v), v / want_s[..., None]).reshape(rows, -1)[:, :cols]
    assert torch.equal(s.nan_to_num(nan=-1.0), want_s.nan_to_num(nan=-1.0))
    if out == "int8":
        assert torch.equal(q, v.nan_to_num(nan=0.0).round().clamp(-127, 127).to(torch.int8))
    else:
        want = v.clamp(-448, 448).to(torch.float8_e4m3fn).float()      # (clamp hands NaN on)
        assert torch.equal(q.float().nan_to_num(nan=-1e9), want.nan_to_num(nan=-1e9))
    return y, s


@pytest.mark.parametrize("rows,cols", [(3, 97), (5, 4096), (301, 1000), (1400, 512), (2, 32768), (299, 8192), (2100, 8192)])
@pytest.mark.parametrize("dtype,weight", [("bf16", "bf16"), ("f32", "f32"), ("f16", "f32")])
@pytest.mark.parametrize("out,group", [("e4m3", 0), ("e4m3", 128), ("e4m3", 32), ("int8", 0), ("int8", 64)])
def test_rms_norm_codes_are_y_over_s_rounded(rows, cols, dtype, weight, out, group):
    torch.manual_seed(rows + cols)
    x = torch.randn(rows, cols, device="cuda").to(TYPES[dtype][0])
    check_codes(x, (1 + 0.3 * torch.randn(cols, device="cuda")).to(TYPES[weight][0]), out, group)


@pytest.mark.parametrize("cols", [96, 256, 333])
@pytest.mark.parametrize("out,group", [("e4m3", 0), ("e4m3", 32), ("int8", 128)])
@pytest.mark.parametrize("size,weight", [(1e-12, 1e-27), (1e-15, 3e-24), (1e4, 5e37), (1e10, 1e30), (1e15, 1e-30), (1e-10, 1e30)])
def test_rms_norm_codes_at_the_ends_of_the_range(cols, out, group, size, weight):
    """x * weight leaves the normal f32 values, y does not (eps = 0: the row's factor is 1 / its size)."""
    torch.manual_seed(cols)
    x = size * torch.randn(4, cols, device="cuda").clamp(-4, 4)
    w = weight * (1 + 0.2 * torch.rand(cols, device="cuda"))
    y, s = check_codes(x, w, out, group, 0.0)
    assert y.isfinite().all() and s.isfinite().all() and (s > 0).all()
