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


@pytest.mark.parametrize("cols", [33, 40, 95, 200, 1001])
@pytest.mark.parametrize("out,group", [("e4m3", 0), ("e4m3", 32), ("int8", 128)])
def test_rms_norm_infinite_weight_in_the_last_column(cols, out, group):
    """The last group's scale is infinite, as the formula says, and not NaN; other groups have theirs."""
    torch.manual_seed(cols)
    x, w = torch.randn(3, cols, device="cuda"), 1 + torch.rand(cols, device="cuda")
    w[-1] = float("inf")
    y, s = check_codes(x, w, out, group)
    assert y[:, -1].isinf().all() and s[:, -1].isinf().all() and s[:, :-1].isfinite().all()


@pytest.mark.parametrize("cols", [33, 40, 200, 1001])
def test_rms_norm_squares_that_vanish(cols):
    """eps = 0 and entries whose squares are below f32: the factor is infinite and so is y; no column beyond the last makes a NaN of the scale."""
    y, s = check_codes(1e-25 * (1 + torch.rand(3, cols, device="cuda")), torch.ones(cols, device="cuda"), "e4m3", 128, 0.0)
    assert y.isinf().all() and s.isinf().all()


# ---- mixture of experts

def one_expert(hidden, inner, dtype, g, u, d):
    """A layer of one expert from integer weights -7..7 (g, u: inner x hidden, d: hidden x inner), all scales 1; returns call(x) -> y."""
    boxes = [pack((torch.as_tensor(w).reshape(1, *w.shape).numpy() + 8).astype(np.uint8), torch.ones(1, w.shape[0], 1), None, 0)[1] for w in (g, u, d)]
    plan = mom.mom_moe_plan(hidden, inner, 1, 1, TYPES[dtype][1], mom.F32, 0, mom.F32, False, True)
    r = torch.zeros(1, hidden, device="cuda")

    def call(x):
        y = torch.empty_like(x)
        room = plan.workspace_bytes(x.shape[0])
        ws = torch.full((room,), 255, dtype=torch.uint8, device="cuda")
        plan.execute(x.shape[0], ptr(x), ptr(r), *map(ptr, boxes), ptr(y), None, None, ptr(ws), room, stream())
        torch.cuda.synchronize()
        assert plan.device_status() == (0, 0)
        return y
    return call


def silu(a):
    return a / (1 + np.exp(-a))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("tokens", [3, 64])
def test_moe_holds_h_in_32_bits(tokens, dtype):
    """h_0 = silu(x_0) * 7 x_0 and h_1 = silu(x_0) * (7 x_0 + x_1) with x_1 = x_0 / 1024 nearly cancel in y = 7 h_0 - 7 h_1 = -7 silu(x_0) x_1."""
    torch.manual_seed(tokens)
    g, u = np.zeros((2, 64), np.int64), np.zeros((2, 64), np.int64)
    g[:, 0], u[:, 0], u[1, 1] = 1, 7, 1
    x = torch.zeros(tokens, 64, device="cuda")
    x[:, 0] = 0.5 + 3.5 * torch.rand(tokens, device="cuda")
    x[:, 1] = x[:, 0] * 2.0 ** -10
    x = x.to(TYPES[dtype][0])
    y = host(one_expert(64, 2, dtype, g, u, np.tile([7, -7], (64, 1)))(x))
    v = host(x)
    h = silu(v[:, 0]) * 7 * v[:, 0]
    want = (-7 * silu(v[:, 0]) * v[:, 1])[:, None]
    # silu is the same number in both (16 u covers exp, sum, quotient); 7 x_0 + x_1, the product with silu and 7 h are rounded once each, as is the sum
    bound = 16 * ref.U32 * np.abs(want) + (2 * 7 * 4 * ref.U32 * h)[:, None]
    assert np.all(np.abs(y - want) <= bound + ref.UNIT[dtype] * (np.abs(want) + bound) + ref.TINY[dtype])


@pytest.mark.parametrize("tokens", [1, 5, 8, 40])
def test_moe_f32_keeps_every_bit(tokens):
    """One entry of x that is not zero, one row of G and U: y = 7 silu(x) * 7 x, in which every bit of x and of h shows."""
    torch.manual_seed(tokens)
    x = torch.zeros(tokens, 128, device="cuda")
    at = torch.arange(tokens) * 29 % 128
    v = (0.5 + 3.5 * torch.rand(tokens, device="cuda")) * torch.where(torch.arange(tokens, device="cuda") % 3 == 0, -1.0, 1.0)
    v[0] = 2 - 2.0 ** -23
    x[torch.arange(tokens), at] = v
    y = host(one_expert(128, 1, "f32", np.full((1, 128), 1), np.full((1, 128), 7), np.full((128, 1), 7))(x))
    a = host(v)
    want = (49 * silu(a) * a)[:, None]
    # exp to 2 units at an argument that is exact, sum, quotient, product: 8 u; 7 x and 7 h are summed from three terms, each sum cut at 2 u: 6 u each
    assert np.all(np.abs(y - want) <= 24 * ref.U32 * np.abs(want))


def test_moe_first_call_on_a_side_stream():
    """The first execute of a plan, on a stream that does not wait for the default one, while that one is busy: right, and the same bits as later calls."""
    rng = np.random.default_rng(2)
    side = torch.cuda.Stream()
    codes = [weights(rng, 6, *shape, 32, "bf16", False) for shape in ((96, 128), (96, 128), (128, 96))]
    boxes = [pack(*c, 32)[1] for c in codes]
    x, r = torch.randn(9, 128, device="cuda").to(torch.bfloat16), torch.randn(6, 128, device="cuda").to(torch.bfloat16) / 11
    want, ids, _, bound, _, gap = ref.moe(host(x), host(r), *(dense(*c, 32) for c in codes), 2, True)
    busy, got = torch.randn(8192, 8192, device="cuda"), []
    big = torch.empty(1 << 28, device="cuda")
    torch.cuda.synchronize()
    for _ in range(4):
        plan = mom.mom_moe_plan(128, 96, 6, 2, mom.BF16, mom.BF16, 32)
        room = plan.workspace_bytes(9)
        ws, y = torch.empty(room, dtype=torch.uint8, device="cuda"), torch.empty_like(x)
        which = torch.empty(9, 2, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        for _ in range(8):                                   # some milliseconds of ordinary work on the default stream
            big.zero_()
            busy @ busy
        for _ in range(2):
            plan.execute(9, ptr(x), ptr(r), *map(ptr, boxes), ptr(y), ptr(which), None, ptr(ws), room, side.cuda_stream)
            with torch.cuda.stream(side):
                got.append(y.clone())
            side.synchronize()
            assert np.array_equal(which.cpu().numpy(), ids)
        torch.cuda.synchronize()
        assert plan.device_status() == (0, 0)
    assert gap > 1e-5 and all(torch.equal(g, got[0]) for g in got)
    assert np.all(np.abs(host(got[0]) - want) <= bound + ref.UNIT["bf16"] * (np.abs(want) + bound))


@pytest.mark.parametrize("cols", [2304, 4099, 5120, 7424, 8192, 8448, 10496, 12544, 16384])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rms_norm_widths_of_many_rows(cols, dtype):
    """However a launch cuts its rows (by width and output), the codes come from the y of the float output."""
    torch.manual_seed(cols)
    check_codes(torch.randn(320, cols, device="cuda").to(TYPES[dtype][0]), 1 + 0.3 * torch.randn(cols, device="cuda"), "e4m3", 128)


# ---- product with 4-bit weights, on both sides of the choice of kernel (more than eight tokens: tcgen05)

@pytest.mark.parametrize("tokens", [1, 2, 5, 8, 9, 20])
@pytest.mark.parametrize("cols", [128, 1003])
@pytest.mark.parametrize("zeros", [False, True])
def test_w4_product_f32_keeps_every_bit(tokens, cols, zeros):
    """One entry a token that is not zero, all scales 1: the three terms of an entry times a code are summed, each sum cut at 2^-23 at most."""
    torch.manual_seed(tokens + cols)
    codes, s, z = weights(np.random.default_rng(tokens), 1, 48, cols, 32, "f32", zeros)
    s = torch.ones_like(s)
    d, box = pack(codes, s, z, 32)
    x = torch.zeros(tokens, cols, device="cuda")
    v = (0.5 + 3.5 * torch.rand(tokens, device="cuda")) * 2.0 ** torch.randint(-60, 60, (tokens,), device="cuda")
    v[0] = -(2 - 2.0 ** -23)
    x[torch.arange(tokens), torch.arange(tokens) * 37 % cols] = v
    y = torch.empty(tokens, 48, device="cuda")
    mom.mom_w4_product(mom.mom_w4_product_desc(d, tokens, mom.F32, mom.F32), ptr(box), ptr(x), None, None, ptr(y), stream())
    torch.cuda.synchronize()
    want = host(x) @ dense(codes, s, z, 32)[0].T
    assert np.all(np.abs(host(y) - want) <= 2.0 ** -22 * np.abs(want))


@pytest.mark.parametrize("tokens", [1, 3, 5, 8, 9, 11, 33])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_w4_product_special_values(tokens, kind):
    """NaN and infinities stay in their token, also in the last one, whose row stands in for tokens that are not there; the others keep their bits."""
    torch.manual_seed(tokens)
    codes, s, z = weights(np.random.default_rng(4), 1, 40, 96, 32, "f32", False)
    codes[codes == 8] = 9                               # no weight is zero
    d, box = pack(codes, s, z, 32)
    w = torch.from_numpy(dense(codes, s, z, 32)[0]).cuda()
    clean = torch.randn(tokens, 96, device="cuda").to(TYPES[kind][0])
    p = mom.mom_w4_product_desc(d, tokens, TYPES[kind][1], mom.F32)

    def product(x):
        y = torch.full((tokens, 40), 5.0, device="cuda")
        mom.mom_w4_product(p, ptr(box), ptr(x), None, None, ptr(y), stream())
        torch.cuda.synchronize()
        return y
    y0 = product(clean)
    for at in sorted({0, tokens // 2, tokens - 1}):
        for value, col in ((float("nan"), 3), (float("inf"), 70), (float("-inf"), 1)):
            x = clean.clone()
            x[at, col] = value
            y = product(x)
            others = [i for i in range(tokens) if i != at]
            assert torch.equal(y[others], y0[others])
            if value != value:
                assert y[at].isnan().all()
            else:
                assert torch.equal(y[at], torch.sign(w[:, col]).float() * value)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("tokens", [2, 10])
def test_moe_special_tokens_keep_the_others_bits(tokens, dtype):
    """A router of zeros sends every token to the first experts, whatever it holds, so that nothing is dealt out otherwise: the other tokens have the same bits."""
    torch.manual_seed(tokens)
    rng = np.random.default_rng(tokens)
    boxes = [pack(*weights(rng, 5, *shape, 32, "bf16", False), 32)[1] for shape in ((64, 128), (64, 128), (128, 64))]
    t, kind = TYPES[dtype]
    r = torch.zeros(5, 128, device="cuda", dtype=t)
    plan = mom.mom_moe_plan(128, 64, 5, 2, kind, kind, 32)
    room = plan.workspace_bytes(tokens)
    ws = torch.empty(room, dtype=torch.uint8, device="cuda")

    def layer(x):
        y, ids = torch.empty_like(x), torch.empty(tokens, 2, dtype=torch.int32, device="cuda")
        plan.execute(tokens, ptr(x), ptr(r), *map(ptr, boxes), ptr(y), ptr(ids), None, ptr(ws), room, stream())
        torch.cuda.synchronize()
        assert plan.device_status() == (0, 0) and ids.cpu().tolist() == [[0, 1]] * tokens
        return y
    x = torch.randn(tokens, 128, device="cuda").to(t)
    y0 = layer(x)
    for at, value in ((tokens - 1, float("nan")), (0, float("inf")), (tokens // 2, float("-inf"))):
        special = x.clone()
        special[at, 5] = value
        y = layer(special)
        others = [i for i in range(tokens) if i != at]
        assert torch.equal(y[others], y0[others]) and y[at].isnan().all()


@pytest.mark.parametrize("hidden,inner,count,top_k", [(256, 64, 4, 2), (48, 2000, 9, 3)], ids=["whole rows of D", "rows of D shared by CTAs"])
def test_moe_wait_that_runs_out(hidden, inner, count, top_k):
    """The self-test's missing arrival: y is NaN and never a number that may be wrong, the status tells of it once, and the next execute has its bits again."""
    torch.manual_seed(inner)
    rng = np.random.default_rng(inner)
    boxes = [pack(*weights(rng, count, *shape, 32, "bf16", False), 32)[1] for shape in ((inner, hidden), (inner, hidden), (hidden, inner))]
    x, r = torch.randn(40, hidden, device="cuda").to(torch.bfloat16), torch.randn(count, hidden, device="cuda").to(torch.bfloat16)
    plan = mom.mom_moe_plan(hidden, inner, count, top_k, mom.BF16, mom.BF16, 32)
    room = plan.workspace_bytes(40)
    ws = torch.empty(room, dtype=torch.uint8, device="cuda")

    def layer():
        y = torch.zeros_like(x)
        plan.execute(40, ptr(x), ptr(r), *map(ptr, boxes), ptr(y), None, None, ptr(ws), room, stream())
        torch.cuda.synchronize()
        return y
    want = layer()
    assert plan.device_status() == (0, 0) and want.isfinite().all()
    plan.probe_wait_timeout(3.0)
    assert layer().isnan().all()
    assert torch.equal(layer(), want)                        # also before the status has been read
    code, detail = plan.device_status()
    assert code == mom.ERR_DEVICE_TIMEOUT and detail in (1, 2, 3)
    assert plan.device_status() == (0, 0)
    assert torch.equal(layer(), want) and plan.device_status() == (0, 0)
    for bad in (0.0, -1.0, 1001.0):
        with pytest.raises(mom.MomError):
            plan.probe_wait_timeout(bad)


def normwise(got, want):
    return np.linalg.norm(host(got) - want) / np.linalg.norm(want)


@pytest.mark.parametrize("tokens,rows,cols,group,zeros", [(1, 512, 4096, 128, False), (8, 300, 2048, 32, False), (7, 400, 5003, 64, True), (3, 200, 9000, 0, False)])
def test_w4_product_f32_is_right_to_the_last_unit(tokens, rows, cols, group, zeros):
    """Normal values, up to eight tokens: normwise off by at most one unit of f32, 2^-23."""
    torch.manual_seed(cols)
    codes, s, z = weights(np.random.default_rng(cols), 1, rows, cols, group, "f32", zeros)
    d, box = pack(codes, s, z, group)
    x, y = torch.randn(tokens, cols, device="cuda"), torch.empty(tokens, rows, device="cuda")
    mom.mom_w4_product(mom.mom_w4_product_desc(d, tokens, mom.F32, mom.F32), ptr(box), ptr(x), None, None, ptr(y), stream())
    torch.cuda.synchronize()
    assert normwise(y, ref.product(host(x), dense(codes, s, z, group)[0])) <= 2.0 ** -23


@pytest.mark.parametrize("tokens,hidden,inner,count,top_k,group", [(5, 1001, 333, 10, 3, 32), (20, 320, 558, 16, 3, 64), (9, 1024, 512, 8, 2, 128)])
def test_moe_f32_is_right_to_the_last_units(tokens, hidden, inner, count, top_k, group):
    """Three such products in a row: at most three units."""
    torch.manual_seed(hidden)
    rng = np.random.default_rng(hidden)
    parts = [weights(rng, count, *shape, group, "f32", False) for shape in ((inner, hidden), (inner, hidden), (hidden, inner))]
    boxes = [pack(*p, group)[1] for p in parts]
    x, r = torch.randn(tokens, hidden, device="cuda"), torch.randn(count, hidden, device="cuda") / hidden ** 0.5
    want, ids, _, _, _, gap = ref.moe(host(x), host(r), *(dense(*p, group) for p in parts), top_k, True)
    plan = mom.mom_moe_plan(hidden, inner, count, top_k, mom.F32, mom.F32, group, mom.F32)
    room = plan.workspace_bytes(tokens)
    ws, y = torch.empty(room, dtype=torch.uint8, device="cuda"), torch.empty_like(x)
    plan.execute(tokens, ptr(x), ptr(r), *map(ptr, boxes), ptr(y), None, None, ptr(ws), room, stream())
    torch.cuda.synchronize()
    assert plan.device_status() == (0, 0) and gap > 1e-5
    assert normwise(y, want) <= 3 * 2.0 ** -23


@pytest.mark.parametrize("tokens,rows,cols,group", [(64, 512, 4096, 128), (40, 300, 8192, 0), (20, 700, 5003, 64)])
def test_w4_product_of_many_f32_tokens_is_right_to_two_units(tokens, rows, cols, group):
    """Normal values, more than eight tokens (one accumulator for all terms): normwise off by at most two units of f32, 2^-22."""
    torch.manual_seed(cols)
    codes, s, z = weights(np.random.default_rng(cols), 1, rows, cols, group, "f32", False)
    d, box = pack(codes, s, z, group)
    x, y = torch.randn(tokens, cols, device="cuda"), torch.empty(tokens, rows, device="cuda")
    mom.mom_w4_product(mom.mom_w4_product_desc(d, tokens, mom.F32, mom.F32), ptr(box), ptr(x), None, None, ptr(y), stream())
    torch.cuda.synchronize()
    assert normwise(y, ref.product(host(x), dense(codes, s, z, group)[0])) <= 2.0 ** -22
