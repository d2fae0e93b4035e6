"""The microscaled operators on the GPU against their definitions in 64 bits (mx_reference)."""
import ctypes

import pytest
import torch

import mx_reference as R
import paper_2604_14156_b200 as cs
from paper_2604_14156_b200 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(shape, generator=g, device=DEV)


# ---- quantisation ------------------------------------------------------------------------------------

def check_quantized(w, transpose):
    codes, scales = cs.cs_mx_quantize(w, transpose=transpose)
    m = w.t() if transpose else w
    v, byte = R.quantize4(m)
    assert codes.shape == (m.shape[0], 16 * byte.shape[1]) and scales.shape == byte.shape
    assert torch.equal(scales.view(torch.uint8), byte)
    assert torch.equal(R.codes4(codes), v)
    back = cs.cs_mx_dequantize(codes, scales, m.shape[1], w.dtype)
    # values are exact in both types but for 2^128, which magnitudes above 3.5 2^126 round to: an infinity
    exact = R.values4(codes, scales)[:, :m.shape[1]]
    want = exact.to(w.dtype).double()
    assert torch.equal(want[exact.abs() < 2.0 ** 128], exact[exact.abs() < 2.0 ** 128])
    assert torch.equal(torch.isnan(back), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(back.double()), torch.nan_to_num(want))


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (32, 1), (3, 33), (31, 64), (129, 8), (257, 100), (64, 1000), (300, 514), (1031, 2051), (256, 64)])
def test_quantize_matches_definition(rows, cols, dtype, transpose):
    w = randn(gen(rows * 7 + cols), rows, cols) * torch.exp(3 * randn(gen(5), rows, 1))
    check_quantized(w.to(dtype), transpose)


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_extreme_values(dtype, transpose):
    w = torch.zeros((96, 96), device=DEV)
    w[0, 0] = float("nan")
    w[33, 1] = float("inf")
    w[34, 40] = -float("inf")
    w[35] = torch.finfo(torch.float32).tiny * randn(gen(1), 96)
    w[36] = torch.finfo(torch.bfloat16).max
    w[37] = 2.0 ** -133 * torch.arange(96, device=DEV)
    w[38, ::2], w[38, 1::2] = 6.0, -0.25            # a tie between 0 and 0.5: 0
    w[39] = torch.tensor([0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -2.5], device=DEV).repeat(12)    # ties of every binade
    w[40] = torch.nextafter(torch.tensor(6.0), torch.tensor(7.0)).item() if dtype == torch.float32 else 6.03125
    w[41, 3] = -0.0
    w[70:, 70:] = 3e38
    check_quantized(w.to(dtype), transpose)


@pytest.mark.parametrize("transpose", [False, True])
def test_quantize_strided_and_unaligned(transpose):
    base = randn(gen(3), 200, 333).bfloat16()
    for view in (base[:, 1:130], base[3:150, 8:136], base[::2, :64], base[5:6, 7:300]):
        check_quantized(view, transpose)
    out = torch.full((40, 100), 7.0, device=DEV)
    codes, scales = cs.cs_mx_quantize(base[:40, :70])
    cs.cs_mx_dequantize(codes, scales, 70, out=out[:, 10:80])
    assert torch.equal(out[:, 10:80].double(), R.values4(codes, scales)[:, :70])
    assert (out[:, :10] == 7).all() and (out[:, 80:] == 7).all()


@pytest.mark.parametrize("cols", [2 ** 31 - 1, 2 ** 31 - 8])
def test_quantize_the_longest_row(cols):
    """A row whose blocks, but not whose rounded-up length, can be counted in 32 bits."""
    w = torch.zeros((1, cols), dtype=torch.bfloat16, device=DEV)
    w[0, :100] = randn(gen(11), 100).bfloat16()
    w[0, -100:] = randn(gen(12), 100).bfloat16()
    codes, scales = cs.cs_mx_quantize(w)
    nb = 2 ** 26
    assert scales.shape == (1, nb) and codes.shape == (1, 16 * nb)
    for at, n in ((0, 128), ((nb - 4) * 32, cols - (nb - 4) * 32)):
        v, byte = R.quantize4(w[:, at:at + n])
        assert torch.equal(scales.view(torch.uint8)[:, at // 32:at // 32 + 4], byte)
        assert torch.equal(R.codes4(codes[:, at // 2:at // 2 + 64]), v)
    assert int(scales.view(torch.uint8)[:, 4:-4].max()) == 0 and int(codes[:, 64:-64].max()) == 0
    back = torch.full((1, cols), 7.0, dtype=torch.bfloat16, device=DEV)
    cs.cs_mx_dequantize(codes, scales, cols, out=back)
    assert torch.equal(back[0, -64:].double(), R.values4(codes[:, -256:], scales[:, -16:])[0, :cols - (nb - 16) * 32][-64:])
    assert int(torch.count_nonzero(back[:, 128:-128])) == 0
    del w, codes, scales, back
    binding._matrix_templates.clear()
    torch.cuda.empty_cache()


def test_quantize_refusals():
    w = randn(gen(1), 64, 64)
    with pytest.raises(ValueError):
        cs.cs_mx_quantize(w.t())
    with pytest.raises(ValueError):
        cs.cs_mx_quantize(w[:0])
    with pytest.raises(TypeError):
        cs.cs_mx_quantize(w.half())
    codes, scales = cs.cs_mx_quantize(w)
    with pytest.raises(ValueError):
        cs.cs_mx_dequantize(codes, scales, 65)
    with pytest.raises(TypeError):
        cs.cs_mx_dequantize(codes, scales.float(), 64)
    with pytest.raises(ValueError):
        cs.cs_mx_quantize(w, codes=codes[:, :16])


# ---- norm ----------------------------------------------------------------------------------------------

def check_norm(x, gamma, delta, eps, got, rows=None):
    h, q, s, n = got
    B, d = x.shape
    want_h = x if delta is None else (x.float() + delta.float()).to(x.dtype)
    assert torch.equal(torch.nan_to_num(h.double(), nan=1e300), torch.nan_to_num(want_h.double(), nan=1e300))
    f = want_h.double()
    want = f / torch.sqrt(f.square().mean(1, keepdim=True) + eps) * (1 if gamma is None else gamma.double())
    # a row with a NaN is NaN; with an infinity, h / inf is 0 but for the infinity itself, whose block is NaN
    fine = torch.isfinite(want).reshape(B, -1, 32).all(2).repeat_interleave(32, dim=1)
    # h itself is exact; the sum of squares (f32, a tree) enters with half its error, then root, division and two products: 2^-20 in all
    err = 2.0 ** -20 * want.abs()
    if n is not None:
        assert ((n.double() - want).abs() <= err)[fine].all() and torch.isnan(n[torch.isnan(want)]).all()
    scale = R.untiles(s, B, d // 32)
    value = q.double() * scale.repeat_interleave(32, dim=1)
    assert torch.isnan(value[~fine]).all()
    want = torch.where(fine, want, torch.zeros_like(want))
    _, step, _ = R.round8(want)
    # half a step of e4m3; a scale whose block's largest lies on the border may be the next one, which doubles the steps of the smallest elements
    top = want.abs().reshape(B, d // 32, 32).amax(-1)
    want_scale = R.two_to(R.exponent(top, 448.0))
    lo, hi = R.two_to(R.exponent(top * (1 - 2.0 ** -20), 448.0)), R.two_to(R.exponent(top * (1 + 2.0 ** -20), 448.0))
    good = fine[:, ::32]
    assert ((scale >= lo) & (scale <= hi))[good].all()
    step = torch.where((lo < hi).repeat_interleave(32, dim=1), 2 * step, step)
    assert ((value - want).abs() <= step / 2 + 2.0 ** -20 * want.abs())[fine].all()
    # most scales are those of the definition
    assert (scale == want_scale)[good].double().mean() > 0.99
    # padding of the last tile of 128 rows
    byte = torch.zeros((B, d // 32), dtype=torch.uint8, device=x.device)
    pad = R.tiles(byte + 1) == 0
    assert (s.view(torch.uint8)[pad] == 0).all()


@pytest.mark.parametrize("B,d", [(1, 128), (1, 4096), (2, 640), (33, 256), (127, 1152), (128, 384), (129, 5120), (300, 128), (5, 8192), (1025, 512)])
@pytest.mark.parametrize("xt,dt", [(torch.float32, torch.bfloat16), (torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32),
                                   (torch.float32, None), (torch.bfloat16, None)])
def test_norm_matches_definition(B, d, xt, dt):
    g = gen(B + d)
    x = (randn(g, B, d) * torch.exp(2 * randn(g, B, 1)) * (1 + 50 * (randn(g, 1, d) > 2.5))).to(xt)
    delta = None if dt is None else randn(g, B, d).to(dt)
    gamma = None if B == 2 else 1 + 0.2 * randn(g, d)
    plan = cs.Plan(d, 128, 128, 1, 1, 0, "mx4", B, 1e-5)
    before = x.clone()
    got = cs.cs_mx_norm(plan, x, gamma, delta=delta, want_n=B != 33)
    assert torch.equal(x, before)
    check_norm(x, gamma, delta, 1e-5, got)
    assert plan.device_status() == 0
    # in place: the residual stream updated where it stands
    y = x.clone()
    again = cs.cs_mx_norm(plan, y, gamma, delta=delta, x_out=y)
    assert again[0] is y and torch.equal(y, got[0])
    assert torch.equal(again[1].view(torch.uint8), got[1].view(torch.uint8)) and torch.equal(again[2].view(torch.uint8), got[2].view(torch.uint8))
    plan.close()


@pytest.mark.parametrize("B,d", [(700, 5120), (2100, 4096), (400, 8192), (1300, 1152), (2500, 1024), (610, 4224), (9600, 128)])
@pytest.mark.parametrize("xt,dt", [(torch.float32, torch.bfloat16), (torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, None)])
def test_norm_more_rows_than_one_round(B, d, xt, dt):
    """CTAs that take several rows, with a ring of two to eight of them."""
    test_norm_matches_definition(B, d, xt, dt)


def test_norm_rows_of_zeros_nan_and_infinity():
    g = gen(2)
    x = randn(g, 6, 256)
    x[1] = 0
    x[2, 17] = float("nan")
    x[3, 200] = float("inf")
    x[4] = 1e-30
    x[5, 3] = 1e15
    plan = cs.Plan(256, 128, 128, 1, 1, 0, "mx4", 6, 1e-5)
    got = cs.cs_mx_norm(plan, x, None, want_n=True)
    check_norm(x, None, None, 1e-5, got)
    assert (got[1][1].float() == 0).all()
    plan.close()


def check_rounded_exactly(x, gamma, eps, q, s):
    """q and s are the blocks of the true n, but where n is within 2^-42 of itself of the middle of two values, or the block's largest of the scale's border:
    f64 has 2^-51 of n here, the kernel a root of one Newton step from 2^-22 (2^-43) and products whose errors are carried along (2^-46)."""
    f = x.double()
    n = f / torch.sqrt(f.square().mean(1, keepdim=True) + eps) * gamma.double()
    v, step, scale = R.round8(n)
    top = n.abs().reshape(x.shape[0], -1, 32).amax(-1)
    sure = ~((top * (1 + 2.0 ** -42) > 448 * scale) | (top * (1 - 2.0 ** -42) <= 224 * scale))
    got = R.untiles(s, x.shape[0], x.shape[1] // 32)
    assert torch.equal(got[sure], scale[sure])
    sure = sure.repeat_interleave(32, dim=1) & ((n / step - torch.floor(n / step) - 0.5).abs() * step > 2.0 ** -42 * n.abs())
    value = q.double() * got.repeat_interleave(32, dim=1)
    assert torch.equal(value[sure], v[sure]), int((value != v)[sure].sum())
    assert sure.double().mean() > 0.99


@pytest.mark.parametrize("B,d", [(1, 256), (3, 4096), (700, 4096), (700, 5120), (1300, 1152), (2500, 1280)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_rounds_the_true_value(B, d, dtype):
    """Rows of which a few channels hold nearly all of the sum of squares."""
    g = gen(B + d)
    plan = cs.Plan(d, 128, 128, 1, 1, 0, "mx4", B, 1e-5)
    for hot in (1, 31, 1000):
        x = (randn(g, B, d) * (1 + hot * (torch.rand((B, d), generator=g, device=DEV) < 0.01))).to(dtype)
        gamma = 1 + 0.2 * randn(g, d)
        _, q, s, _ = cs.cs_mx_norm(plan, x, gamma)
        check_rounded_exactly(x, gamma, 1e-5, q, s)
    plan.close()


@pytest.mark.parametrize("B,d", [(1, 256), (2, 4096), (700, 4096), (700, 5120), (1300, 1152), (2500, 1280)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_next_to_the_middles(B, d, dtype):
    """gamma chosen so that every n is within a unit or two of f32 of the middle of two e4m3 values, and the blocks' largest as near to a border of the scale."""
    g = gen(3 * B + d)
    x = (randn(g, 1, d) * (1 + 30 * (torch.rand((1, d), generator=g, device=DEV) < 0.01))).to(dtype)
    x[x == 0] = 1
    f = x.double()
    r = 1 / torch.sqrt(f.square().mean(1, keepdim=True) + 1e-5)
    # middles: (8 .. 15 + 1/2) 2^p under a largest of 448, which is 14 2^5
    target = (8.5 + torch.randint(8, (1, d), generator=g, device=DEV)) * 2.0 ** torch.randint(-8, 5, (1, d), generator=g, device=DEV)
    target[:, 5::32] = 448.0
    target *= 2.0 ** torch.randint(-3, 4, (1, d // 32), generator=g, device=DEV).repeat_interleave(32, dim=1)
    gamma = (target.double() / (f * r)).float()
    ulp = 1 + 2.0 ** -23 * torch.randint(-2, 3, (1, d), generator=g, device=DEV)
    gamma = (gamma.double() * ulp).float()[0].contiguous()
    plan = cs.Plan(d, 128, 128, 1, 1, 0, "mx4", B, 1e-5)
    x = x.expand(B, d).contiguous()
    _, q, s, _ = cs.cs_mx_norm(plan, x, gamma)
    check_rounded_exactly(x, gamma, 1e-5, q, s)
    plan.close()


@pytest.mark.parametrize("B,d", [(6, 256), (800, 4096), (2500, 1024), (1300, 1152)])
@pytest.mark.parametrize("xt,dt", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.bfloat16, None)])
def test_norm_rows_of_nan_and_infinity_keep_to_themselves(B, d, xt, dt):
    g = gen(B + 1)
    x, delta = randn(g, B, d).to(xt), None if dt is None else randn(g, B, d).to(dt)
    plan = cs.Plan(d, 128, 128, 1, 1, 0, "mx4", B, 1e-5)
    want = cs.cs_mx_norm(plan, x, None, delta=delta, want_n=True)
    x[1] = 0
    x[2, 17] = float("nan")
    x[B - 2, 200] = float("inf")
    if dt is not None:
        delta[1] = 0
        delta[B // 2, d - 1] = float("nan")
        delta[B - 1, 3] = -float("inf")
    got = cs.cs_mx_norm(plan, x, None, delta=delta, want_n=True)
    check_norm(x, None, delta, 1e-5, got)
    same = torch.ones(B, dtype=torch.bool, device=DEV)
    same[[1, 2, B // 2, B - 2, B - 1]] = False
    for a, b in ((want[0], got[0]), (want[1].view(torch.uint8), got[1].view(torch.uint8)), (want[3], got[3])):
        assert torch.equal(a[same], b[same])
    assert (got[1][1].float() == 0).all() and plan.device_status() == 0
    plan.close()


@pytest.mark.parametrize("B", [1, 70, 900])
def test_norm_reads_a_gamma_that_the_call_ahead_writes(B):
    d = 4096
    g = gen(B)
    plan = cs.Plan(d, 128, 128, 1, 1, 0, "mx4", B, 1e-5)
    x = randn(g, B, d)
    gammas = [cs.cs_mx_quantize(1 + 0.2 * randn(g, 1, d)) for _ in range(2)]
    rows = [cs.cs_mx_dequantize(*q, d, torch.float32) for q in gammas]
    torch.cuda.synchronize()
    want = [cs.cs_mx_norm(plan, x, r[0])[1].view(torch.uint8) for r in rows]
    assert not torch.equal(*want)
    torch.cuda.synchronize()
    row = torch.empty((1, d), device=DEV)
    wrong = torch.zeros((), dtype=torch.int64, device=DEV)
    for i in range(200):
        cs.cs_mx_dequantize(*gammas[i % 2], d, out=row)
        q = cs.cs_mx_norm(plan, x, row[0])[1]
        wrong += (q.view(torch.uint8) != want[i % 2]).sum()
    assert int(wrong) == 0
    plan.close()


def test_norm_refusals():
    plan = cs.Plan(256, 128, 128, 1, 1, 0, "mx4", 4, 1e-5)
    x = randn(gen(1), 4, 256)
    with pytest.raises(TypeError):
        cs.cs_mx_norm(plan, x.half())
    with pytest.raises(ValueError):
        cs.cs_mx_norm(plan, x[:, :128])
    with pytest.raises(ValueError):
        cs.cs_mx_norm(plan, x, delta=x[:2])
    with pytest.raises(TypeError):
        cs.cs_mx_norm(plan, x.cpu())
    with pytest.raises(cs.CSError) as e:
        cs.cs_mx_norm(plan, torch.zeros((5, 256), device=DEV))
    assert e.value.code == 2
    with pytest.raises(cs.CSError) as e:
        cs.cs_mx_norm(plan, torch.zeros(4 * 256 + 1, device=DEV)[1:].view(4, 256))
    assert e.value.code == 3
    other = cs.Plan(256, 128, 128, 1, 1, 0, torch.bfloat16, 4, 1e-5)
    with pytest.raises(cs.CSError) as e:
        cs.cs_mx_norm(other, x)
    assert e.value.code == 3
    plan.close()
    other.close()


# ---- FFN -------------------------------------------------------------------------------------------------

class Problem:
    def __init__(self, B, d, G, k, shared, seed=0, plan_tokens=None):
        g = gen(1000 * seed + B + d + G)
        self.B, self.d, self.G, self.k, self.shared = B, d, G, k, shared
        d_ff = 128 * G
        self.gate, self.up = (cs.cs_mx_quantize(randn(g, d_ff, d) / d ** 0.5) for _ in range(2))
        self.down = cs.cs_mx_quantize((randn(g, d_ff, d) / (128 * k) ** 0.5).bfloat16(), transpose=True)
        self.plan = cs.Plan(d, d_ff, 128, 1, k, 0, "mx4", plan_tokens or B, 1e-5)
        self.layer = cs.MxLayer(self.plan, self.gate, self.up, self.down)
        self.new_inputs(g, B)

    def new_inputs(self, g, B):
        self.B = B
        x = randn(g, B, self.d) * torch.exp(randn(g, B, 1))
        _, self.q, self.s, _ = cs.cs_mx_norm(self.plan, x)
        # rows differ in size: the norm has evened them out, so scale some blocks' bytes
        draw = torch.rand((1 if self.shared else B, self.G), generator=g, device=DEV)
        sup = draw.topk(self.k, dim=1).indices.sort(dim=1).values.to(torch.int32)
        self.support = sup[0].contiguous() if self.shared else sup

    def run(self, **kw):
        return (cs.cs_mx_ffn_shared if self.shared else cs.cs_mx_ffn)(self.plan, self.layer, self.q, self.s, self.support, **kw)

    def operands(self):
        x = self.q.double() * R.untiles(self.s, self.B, self.d // 32).repeat_interleave(32, dim=1)
        return x, R.values4(*self.gate), R.values4(*self.up), R.values4(*self.down)

    def member(self):
        m = torch.zeros((self.support.reshape(-1, self.k).shape[0], self.G), dtype=torch.bool, device=DEV)
        m.scatter_(1, self.support.reshape(-1, self.k).long(), True)
        return m.expand(self.B, self.G).repeat_interleave(128, dim=1)

    def check(self, out):
        want, tol = R.ffn(*self.operands(), self.member())
        off = (out.double() - want).abs()
        assert (off <= tol).all(), float((off / tol).max())
        assert self.plan.device_status() == 0


@pytest.mark.parametrize("d,G", [(128, 1), (640, 3), (1024, 16)])
def test_pack_is_the_documented_order(d, G):
    g = gen(d + G)
    gate, up = (cs.cs_mx_quantize(randn(g, 128 * G, d) * torch.exp(2 * randn(g, 128 * G, 1))) for _ in range(2))
    down = cs.cs_mx_quantize(randn(g, 128 * G, d) * torch.exp(2 * randn(g, 1, d)), transpose=True)
    plan = cs.Plan(d, 128 * G, 128, 1, 1, 0, "mx4", 1, 1e-5)
    got = [t.clone() for t in cs.MxLayer(plan, gate, up, down).tensors]
    kb = d // 128

    def tile_scales(s):           # [tiles, 128, 4] -> tile order
        return torch.cat([R.tiles(x).reshape(1, 512) for x in s])
    # gate_up: group, 128 columns, half of the channels: 64 rows of gate, the same 64 of up
    c = torch.stack([m[0].reshape(G, 2, 64, kb, 64) for m in (gate, up)], 2).permute(0, 4, 1, 2, 3, 5).reshape(-1, 128, 64)
    s = torch.stack([m[1].view(torch.uint8).reshape(G, 2, 64, kb, 4) for m in (gate, up)], 2).permute(0, 4, 1, 2, 3, 5).reshape(-1, 128, 4)
    assert torch.equal(got[0], c.reshape(-1)) and torch.equal(got[1], tile_scales(s).reshape(-1))
    # down: group, 128 rows
    c = down[0].reshape(kb, 128, G, 64).permute(2, 0, 1, 3).reshape(-1, 128, 64)
    s = down[1].view(torch.uint8).reshape(kb, 128, G, 4).permute(2, 0, 1, 3).reshape(-1, 128, 4)
    assert torch.equal(got[2], c.reshape(-1)) and torch.equal(got[3], tile_scales(s).reshape(-1))
    plan.close()


TOKENS = [1, 2, 3, 15, 16, 17, 31, 33, 64, 65, 100, 112, 113, 127, 128, 129, 144, 200, 255, 256, 257, 300, 513]


@pytest.mark.parametrize("B", TOKENS)
def test_ffn_every_batch(B):
    p = Problem(B, 512, 12, 5, False)
    p.check(p.run())
    p.plan.close()


@pytest.mark.parametrize("n", TOKENS + [777, 1025])
def test_ffn_shared_every_length(n):
    p = Problem(n, 384, 9, 4, True)
    p.check(p.run())
    p.plan.close()


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("d,G,k", [(128, 1, 1), (128, 128, 128), (256, 2, 1), (640, 7, 7), (1152, 3, 2), (4096, 86, 22), (8192, 4, 3), (5120, 20, 11), (1280, 128, 1)])
def test_ffn_shapes(d, G, k, shared):
    for B in (1, 5, 64, 140):
        p = Problem(B, d, G, k, shared, seed=3)
        p.check(p.run())
        p.plan.close()


def test_ffn_rows_behind_the_batch_stay_and_scratch_is_reused():
    """Batches of every size through one plan, larger ones first; the output's other rows keep what they held."""
    p = Problem(300, 256, 10, 3, False)
    g = gen(9)
    for B in (300, 7, 129, 1, 40):
        p.new_inputs(g, B)
        out = torch.full((320, p.d), 3.0, dtype=torch.bfloat16, device=DEV)
        p.run(out=out[:B])
        p.check(out[:B])
        assert (out[B:] == 3).all()
    p.plan.close()


@pytest.mark.parametrize("B", [40, 300, 2000])
def test_ffn_output_on_a_16_byte_boundary(B):
    p = Problem(B, 640, 12, 5, False)
    out = torch.full((B * 640 + 16,), 3.0, dtype=torch.bfloat16, device=DEV)
    rows = out[8:8 + B * 640].view(B, 640)
    assert rows.data_ptr() % 32 == 16
    assert torch.equal(p.run(out=rows), p.run())
    p.check(rows)
    assert (out[:8] == 3).all() and (out[-8:] == 3).all()
    p.plan.close()


def test_ffn_scales_of_padding_rows_may_be_anything():
    p = Problem(20, 256, 6, 2, False)
    want = p.run()
    raw = p.s.view(torch.uint8)
    pad = R.tiles(torch.ones((20, 8), dtype=torch.uint8, device=DEV)) == 0
    raw[pad] = 255
    assert torch.equal(p.run(), want)
    p.check(want)
    p.plan.close()


def test_ffn_a_row_of_nan_keeps_to_itself():
    p = Problem(70, 256, 6, 2, False)
    want = p.run()
    q = p.q.view(torch.uint8)
    q[3, 17] = 0x7F
    p.s.view(torch.uint8)[0, 1, 40 % 32, 40 // 32, 2] = 255     # row 40, block 6
    got = p.run()
    bad = torch.zeros(70, dtype=torch.bool, device=DEV)
    bad[3] = bad[40] = True
    assert torch.isnan(got[bad]).all() and torch.equal(got[~bad], want[~bad])
    p.plan.close()


@pytest.mark.parametrize("B", [1, 6, 40])
def test_ffn_invalid_supports_count_for_nothing_and_are_reported(B):
    p = Problem(B, 256, 6, 3, False)
    p.support[0] = torch.tensor([-1, 2, 6], dtype=torch.int32)
    out = p.run()
    assert p.plan.device_status() == 4
    m = p.member_of = torch.zeros((B, p.G), dtype=torch.bool, device=DEV)
    m.scatter_(1, p.support.clamp(0, 5).long(), True)
    m[0] = False
    m[0, 2] = True
    want, tol = R.ffn(*p.operands(), m.repeat_interleave(128, dim=1))
    assert ((out.double() - want).abs() <= tol).all()
    p.support[:] = -5
    assert (p.run() == 0).all() and p.plan.device_status() == 4
    p.support[:] = 1 << 30
    assert (p.run() == 0).all() and p.plan.device_status() == 4
    p.support[:] = torch.tensor([1, 1, 4], dtype=torch.int32)       # a group twice: once
    out = p.run()
    assert p.plan.device_status() == 4
    m[:] = False
    m[:, 1] = m[:, 4] = True
    want, tol = R.ffn(*p.operands(), m.repeat_interleave(128, dim=1))
    assert ((out.double() - want).abs() <= tol).all()
    p.plan.close()


def test_ffn_shared_equals_own_supports_that_are_all_the_same():
    p = Problem(50, 512, 8, 3, True)
    own = cs.cs_mx_ffn(p.plan, p.layer, p.q, p.s, p.support.expand(50, 3).contiguous())
    assert torch.equal(p.run(), own)
    p.plan.close()


def test_ffn_is_deterministic_and_rows_do_not_depend_on_their_neighbours():
    p = Problem(64, 1024, 16, 5, False)
    out = p.run()
    for _ in range(3):
        assert torch.equal(p.run(), out)
    p.plan.close()


def test_ffn_captured_replayed_and_on_two_streams():
    p = Problem(37, 512, 12, 5, False)
    eager = p.run()
    out = torch.zeros_like(eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run(out=out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, eager)
    g = gen(77)
    x = randn(g, 37, 512)
    _, q, s, _ = cs.cs_mx_norm(p.plan, x)
    p.q.view(torch.uint8).copy_(q.view(torch.uint8))
    p.s.view(torch.uint8).copy_(s.view(torch.uint8))
    graph.replay()
    torch.cuda.synchronize()
    p.check(out)
    # two plans, one stream each
    a, b = Problem(5, 512, 12, 5, False, seed=1), Problem(140, 512, 12, 5, False, seed=2)
    torch.cuda.synchronize()
    sa, sb = torch.cuda.Stream(), torch.cuda.Stream()
    outs = []
    for _ in range(20):
        with torch.cuda.stream(sa):
            oa = a.run()
        with torch.cuda.stream(sb):
            ob = b.run()
        outs.append((oa, ob))
    torch.cuda.synchronize()
    a.check(outs[0][0])
    b.check(outs[0][1])
    assert all(torch.equal(oa, outs[0][0]) and torch.equal(ob, outs[0][1]) for oa, ob in outs)
    for x in (p, a, b):
        x.plan.close()


@pytest.mark.parametrize("B,d,G,k", [(1, 4096, 40, 22), (3, 4096, 40, 22), (16, 2048, 16, 7), (40, 4096, 40, 12), (64, 4096, 40, 22), (100, 2048, 16, 7), (128, 1024, 16, 7),
                                     (200, 2048, 40, 12), (300, 1024, 16, 7)])
def test_ffn_many_calls_back_to_back(B, d, G, k):
    """Launches that overlap their predecessors' ends, thousands of times: every result is the first one."""
    ps = [Problem(B, d, G, k, False, seed=s) for s in (4, 5)]
    want = [p.run() for p in ps]
    outs = [torch.zeros_like(w) for w in want]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(10):
            for p, o in zip(ps, outs):
                p.run(out=o)
    wrong = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(100):
        for o in outs:
            o.fill_(7)
        graph.replay()
        for o, w in zip(outs, want):
            wrong += (o != w).sum()
    assert int(wrong) == 0
    for p, o in zip(ps, outs):
        p.check(o)
        p.plan.close()


def test_ffn_large_batches_on_two_streams():
    """Two plans whose batches take the persistent launch, side by side on streams of different priority and beside other work that comes and goes."""
    ps = [Problem(200, 512, 112, 28, False, seed=1), Problem(700, 768, 24, 9, True, seed=2)]
    want = [p.run() for p in ps]
    for p, w in zip(ps, want):
        p.check(w)
    low, high = torch.cuda.Stream.priority_range()
    streams = [torch.cuda.Stream(priority=low), torch.cuda.Stream(priority=high)]
    third, a = torch.cuda.Stream(), randn(gen(8), 2048, 2048)
    outs = [torch.zeros_like(w) for w in want]
    wrong = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(30):
        for o in outs:
            o.fill_(7)
        torch.cuda.synchronize()
        for _ in range(5):
            with torch.cuda.stream(third):
                a @ a
            for p, s, o in zip(ps, streams, outs):
                with torch.cuda.stream(s):
                    p.run(out=o)
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            wrong += (o != w).sum()
    assert int(wrong) == 0
    for p in ps:
        assert p.plan.device_status() == 0
        p.plan.close()


@pytest.mark.parametrize("sms", [16, 64])
@pytest.mark.parametrize("B,d,G,k,shared", [(300, 1024, 40, 12, False), (200, 512, 112, 28, False), (1100, 640, 24, 9, True), (1500, 512, 60, 20, False)])
def test_ffn_large_batches_on_a_part_of_the_device(B, d, G, k, shared, sms):
    """A launch of which some SMs' worth of CTAs has room at a time: its items are done by those that run."""
    green = pytest.importorskip("torch.cuda.green_contexts")
    if not green.SUPPORTED:
        pytest.skip("torch without green contexts")
    p = Problem(B, d, G, k, shared, seed=6)
    want = p.run()
    p.check(want)
    torch.cuda.synchronize()
    part = green.GreenContext.create(sms, 0)
    stream = part.Stream()
    out = torch.zeros_like(want)
    for _ in range(3):
        out.fill_(7)
        torch.cuda.synchronize()
        p.run(out=out, stream=stream)
        stream.synchronize()
        assert p.plan.device_status() == 0
        assert torch.equal(out, want)
    p.plan.close()
    del part        # not before its stream's last use


@pytest.mark.parametrize("B", [100, 600, 3000])
def test_ffn_activations_are_rounded_within_their_bound(B):
    """W_down = 1, so that the output is a^ itself (four significant bits, exact in bf16), and gates that are exact in f32: wherever silu(gate) up is further
    than 2^-20 of itself from the middle of two e4m3 values, and its block's largest from a border of the scale, a^ is the nearest value."""
    g, d = gen(B), 128
    plan = cs.Plan(d, 128, 128, 1, 1, 0, "mx4", B, 1e-5)
    levels = torch.tensor([1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    support = torch.zeros((B, 1), dtype=torch.int32, device=DEV)
    down = cs.cs_mx_quantize(torch.eye(128, device=DEV), transpose=True)
    up_w = torch.zeros((128, d), device=DEV)
    up_w[:, 127] = 1.0
    checked = 0
    for _ in range(1 + 2000000 // (128 * B)):
        # gate = sum over four blocks of 2^-4b x_b w_b: at most 6 + 12 bits
        w = torch.zeros((128, d), device=DEV)
        w[:, 0] = levels[torch.randint(6, (4,), generator=g, device=DEV)].repeat_interleave(32)      # near gates within a block of channels
        for b in (1, 2, 3):
            w[:, 32 * b] = levels[torch.randint(6, (128,), generator=g, device=DEV)] * (1 - 2 * torch.randint(2, (128,), generator=g, device=DEV))
        gate = cs.cs_mx_quantize(w)
        assert torch.equal(R.values4(*gate), w.double())
        layer = cs.MxLayer(plan, gate, cs.cs_mx_quantize(up_w), down)
        x = torch.zeros((B, d), device=DEV)
        for b in range(4):
            x[:, 32 * b] = (1 + torch.randint(8, (B,), generator=g, device=DEV) / 8) * 2.0 ** torch.randint(-2, 3, (B,), generator=g, device=DEV)
        x[:, 0] *= (1 - 2 * (torch.rand((B,), generator=g, device=DEV) < 0.8).float()) * (x[:, 0] <= 12)
        x[:, 127] = 1.0
        q, e = x.to(torch.float8_e4m3fn), 127 - 4 * torch.arange(4, device=DEV).expand(B, 4)
        e = torch.cat((e[:, :3], torch.full((B, 1), 127 - 12, device=DEV)), 1).to(torch.uint8)
        assert torch.equal(q.float(), x)
        real = x.double() * R.two_to(e.long() - 127).repeat_interleave(32, dim=1)
        out = cs.cs_mx_ffn(plan, layer, q, R.tiles(e).view(torch.float8_e8m0fnu), support).double()
        f, u = real @ w.double().t(), real @ up_w.double().t()
        assert torch.equal(f.float().double(), f)
        a = f / (1 + torch.exp(-f)) * u
        v, step, s = R.round8(a)
        near = 2.0 ** -20 * a.abs()
        top = a.abs().reshape(B, -1, 32).amax(-1)
        border = (top * (1 + 2.0 ** -20) > 448 * s) | (top * (1 - 2.0 ** -20) <= 224 * s)
        sure = ((a / step - torch.floor(a / step) - 0.5).abs() * step > near) & ~border.repeat_interleave(32, dim=1)
        assert (out == v)[sure].all(), (f[sure & (out != v)][:4].tolist(), int((sure & (out != v)).sum()))
        checked += int((sure & (v != 0)).sum())
    assert checked > 700000
    assert plan.device_status() == 0
    plan.close()


# the paths that a batch can take: narrow with the list in the launch and with a list kernel; pairs, with the list in the launch (parts of the list, whole
# lists) and with a list kernel
PATHS = [(3, 256, 6, 3, False), (64, 512, 12, 5, False), (128, 384, 40, 20, False), (100, 256, 8, 3, True), (200, 512, 112, 28, False),
         (300, 256, 10, 3, False), (300, 1024, 90, 12, False), (2000, 256, 12, 5, False), (2000, 1280, 10, 4, True), (1500, 512, 128, 40, False)]


@pytest.mark.parametrize("B,d,G,k,shared", PATHS)
def test_ffn_invalid_supports_on_every_path(B, d, G, k, shared):
    p = Problem(B, d, G, k, shared, seed=8)
    good = p.support.clone()
    rows, sup = (1, p.support.view(1, k)) if shared else (B, p.support)
    bad = torch.full((k,), -7, dtype=torch.int32, device=DEV)
    bad[1], bad[2] = G // 2, G + 3
    sup[rows - 1] = bad                      # the last row: one group
    if rows > 2:
        sup[0] = 1 << 30                     # the first: none
        sup[1] = 1                           # the second: one, many times
    out = p.run()
    assert p.plan.device_status() == 4
    m = torch.zeros((rows, G), dtype=torch.bool, device=DEV)
    m.scatter_(1, good.view(rows, k).long(), True)
    m[rows - 1] = False
    m[rows - 1, G // 2] = True
    if rows > 2:
        m[0] = m[1] = False
        m[1, 1] = True
        assert (out[0] == 0).all()
    want, tol = R.ffn(*p.operands(), m.expand(B, G).repeat_interleave(128, dim=1))
    assert ((out.double() - want).abs() <= tol).all()
    p.support.fill_(-5)
    out.fill_(7)
    assert (p.run(out=out) == 0).all() and p.plan.device_status() == 4
    p.support.copy_(good)
    p.check(p.run())                         # nothing of it stays
    p.plan.close()


@pytest.mark.parametrize("B,d,G,k,shared", PATHS)
def test_ffn_rows_do_not_depend_on_their_neighbours(B, d, G, k, shared):
    """Other rows' activations change, also to NaN, and their supports (the union stays, and with it the order of sums): a row's output does not."""
    p = Problem(B, d, G, k, shared, seed=9)
    g = gen(B)
    if not shared:
        p.support[: -(-G // k)] = torch.stack([torch.arange(i, i + k, device=DEV) if i + k <= G else torch.arange(G - k, G, device=DEV)
                                               for i in range(0, G, k)])[:B].to(torch.int32)
    want = p.run()
    stay = torch.rand((B,), generator=g, device=DEV) < 0.5
    stay[: -(-G // k)] = True
    stay[B // 2] = B == 3
    other = ~stay
    _, q, s, _ = cs.cs_mx_norm(p.plan, randn(g, B, d) * 50)
    q = q.view(torch.uint8)
    byte = torch.where(stay[:, None], R.untiles(p.s, B, d // 32), R.untiles(s, B, d // 32))
    q = torch.where(stay[:, None], p.q.view(torch.uint8), q)
    p.q.view(torch.uint8).copy_(q)
    p.s.view(torch.uint8).copy_(R.tiles((torch.log2(byte) + 127).to(torch.uint8)))
    if not shared:
        new = torch.rand((B, G), generator=g, device=DEV).topk(k, dim=1).indices.sort(dim=1).values.to(torch.int32)
        p.support.copy_(torch.where(stay[:, None], p.support, new))
    got = p.run()
    p.check(got)
    assert torch.equal(got[stay], want[stay])
    if other.any():
        r = int(torch.nonzero(other)[-1])
        q = p.q.view(torch.uint8)
        q[r, 17] = 0x7F
        again = p.run()
        same = torch.ones(B, dtype=torch.bool, device=DEV)
        same[r] = False
        assert torch.isnan(again[r]).all() and torch.equal(again[same], got[same])
        q[r, 17] = 0
        p.s.view(torch.uint8)[r // 128, 1, r % 32, r % 128 // 32, 2] = 255
        again = p.run()
        assert torch.isnan(again[r]).all() and torch.equal(again[same], got[same])
    p.plan.close()


@pytest.mark.parametrize("B,d,G,k,shared", PATHS)
def test_ffn_scales_of_padding_rows_on_every_path(B, d, G, k, shared):
    p = Problem(B, d, G, k, shared, seed=10)
    want = p.run()
    pad = R.tiles(torch.ones((B, d // 32), dtype=torch.uint8, device=DEV)) == 0
    p.s.view(torch.uint8)[pad] = 255
    assert torch.equal(p.run(), want)
    p.check(want)
    p.plan.close()


@pytest.mark.parametrize("B,d,G,k,shared", [(1, 4096, 40, 22, False), (16, 2048, 16, 7, False), (64, 1024, 40, 12, False), (128, 384, 40, 20, False), (100, 256, 8, 3, True)])
def test_ffn_small_batches_on_a_part_of_the_device(B, d, G, k, shared):
    """Clusters, and down CTAs that start beside gate/up's, where 16 SMs are all there is."""
    test_ffn_large_batches_on_a_part_of_the_device(B, d, G, k, shared, 16)


def test_plans_created_by_several_threads_at_once():
    """The FFN's launch shapes come from the plan: plans created side by side give what one created alone gives."""
    import threading
    p = Problem(64, 1024, 16, 5, False, seed=7)
    want = p.run()
    torch.cuda.synchronize()
    got, errors = [], []

    def work():
        try:
            for _ in range(5):
                plan = cs.Plan(1024, 2048, 128, 1, 5, 0, "mx4", 64, 1e-5)
                stream = torch.cuda.Stream()
                with torch.cuda.stream(stream):
                    got.append(cs.cs_mx_ffn(plan, p.layer, p.q, p.s, p.support))
                stream.synchronize()
                plan.close()
        except Exception as e:
            errors.append(e)
    threads = [threading.Thread(target=work) for _ in range(6)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors and len(got) == 30 and all(torch.equal(o, want) for o in got)
    p.plan.close()


def test_ffn_refusals():
    p = Problem(8, 256, 4, 2, False)
    with pytest.raises(ValueError):
        p.run(out=torch.zeros((7, 256), dtype=torch.bfloat16, device=DEV))
    with pytest.raises(TypeError):
        p.run(out=torch.zeros((8, 256), device=DEV))
    with pytest.raises(ValueError):
        cs.cs_mx_ffn(p.plan, p.layer, p.q, p.s, p.support[:, :1].contiguous())
    with pytest.raises(TypeError):
        cs.cs_mx_ffn(p.plan, p.layer, p.q.float(), p.s, p.support)
    with pytest.raises(ValueError):
        cs.cs_mx_ffn(p.plan, p.layer, p.q, p.s.view(-1), p.support)
    with pytest.raises(ValueError):
        cs.MxLayer(p.plan, p.gate, p.up, p.gate)
    big = torch.zeros((9, 256), dtype=torch.float8_e4m3fn, device=DEV)
    with pytest.raises(cs.CSError) as e:
        cs.cs_mx_ffn(p.plan, p.layer, big, p.s, torch.zeros((9, 2), dtype=torch.int32, device=DEV))
    assert e.value.code == 2
    lib, layer = p.plan.lib, p.layer
    args = [layer.ref, p.q.data_ptr(), p.s.data_ptr(), p.support.data_ptr(), 8, torch.zeros((8, 256), dtype=torch.bfloat16, device=DEV).data_ptr(), None]
    for i in (1, 2, 3, 5):
        broken = list(args)
        broken[i] = None
        assert lib.cs_mx_ffn(p.plan.handle, *broken) == 1
    for i in (1, 2, 5):
        broken = list(args)
        broken[i] += 8
        assert lib.cs_mx_ffn(p.plan.handle, *broken) == 3
    bad = binding._MxLayer(layer.c.gate_up_codes + 16, layer.c.gate_up_scales, layer.c.down_codes, layer.c.down_scales)
    assert lib.cs_mx_ffn(p.plan.handle, ctypes.byref(bad), *args[1:]) == 3
    # a plan of one kind does not take the other kind's calls
    other = cs.Plan(256, 512, 128, 1, 2, 0, torch.bfloat16, 8, 1e-5)
    assert lib.cs_mx_ffn(other.handle, *args) == 3
    w = torch.zeros((512, 256), dtype=torch.bfloat16, device=DEV)
    plain = cs.Layer(other, torch.zeros((1, 256), device=DEV), torch.zeros((1, 4), device=DEV), w, w, w, 1.0)
    h = torch.zeros((8, 256), device=DEV)
    calls = [lambda: cs.cs_ffn_exec(p.plan, plain, h, p.support), lambda: cs.cs_layer_step(p.plan, plain, h),
             lambda: cs.cs_layer_step_ex(p.plan, plain, h, cs.StepOptions(p.plan, 8)),
             lambda: cs.cs_layer_step_host(p.plan, plain, h.cpu(), h.cpu()),
             lambda: cs.cs_layer_step_fallback(p.plan, p.plan, plain, h, 0.5),
             lambda: cs.cs_ffn_exec_shared(p.plan, plain, h.bfloat16(), p.support[0].contiguous()), lambda: p.plan.set_speculative(1)]
    for call in calls:
        with pytest.raises(cs.CSError) as e:
            call()
        assert e.value.code == 3
    p.plan.close()
    other.close()


# ---- together -----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("B", [1, 9, 48])
def test_two_layers_of_a_decode_step(B, oracle):
    """norm -> sketch -> recovery -> FFN -> the next layer's norm, each stage against its definition on what the stage before really gave."""
    import numpy as np
    d, G, m, k, T = 512, 16, 16, 5, 12
    g = gen(B)
    plan = cs.Plan(d, 128 * G, 128, m, k, T, "mx4", B, 1e-5)
    x, delta = randn(g, B, d), None
    for _ in range(2):
        gate, up = (cs.cs_mx_quantize(randn(g, 128 * G, d) / d ** 0.5) for _ in range(2))
        down = cs.cs_mx_quantize(randn(g, 128 * G, d) / (128 * k) ** 0.5, transpose=True)
        layer = cs.MxLayer(plan, gate, up, down)
        S, Phi, gamma = randn(g, m, d) / d ** 0.5, randn(g, m, G) / m ** 0.5, 1 + 0.1 * randn(g, d)
        mu = float(1 / torch.linalg.matrix_norm(Phi.double(), 2) ** 2)
        torch.cuda.synchronize()
        before = x.clone()
        x, q, s, n = cs.cs_mx_norm(plan, x, gamma, delta=delta, want_n=True, x_out=x)
        y = cs.cs_sketch(plan, S, n)
        support, z, resid = cs.cs_recover(plan, Phi, mu, y)
        out = cs.cs_mx_ffn(plan, layer, q, s, support)
        assert plan.device_status() == 0
        check_norm(before, gamma, delta, 1e-5, (x, q, s, n))
        # f32 sums of d products
        assert ((y.double() - n.double() @ S.double().t()).abs() <= 2.0 ** -18 * (n.double().abs() @ S.double().abs().t())).all()
        for t in range(B):
            ref = oracle.iht(Phi.cpu(), y[t].cpu(), k, T, mu)
            assert np.array_equal(support[t].cpu().numpy(), ref.support) or ref.min_gap <= 1e-4
        member = torch.zeros((B, G), dtype=torch.bool, device=DEV).scatter_(1, support.long(), True).repeat_interleave(128, dim=1)
        xq = q.double() * R.untiles(s, B, d // 32).repeat_interleave(32, dim=1)
        want, tol = R.ffn(xq, R.values4(*gate), R.values4(*up), R.values4(*down), member)
        assert ((out.double() - want).abs() <= tol).all()
        delta = out
    plan.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_dequantised_weights_go_straight_into_the_other_ffn(dtype):
    """All three matrices dequantised in front of the call that takes them as parameters, into the same place for two layers in turn."""
    d, G, k, B = 256, 6, 2, 3
    g = gen(31)
    plan = cs.Plan(d, 128 * G, 128, 1, k, 0, dtype, B, 1e-5)
    sources = [[cs.cs_mx_quantize(randn(g, 128 * G, d) / 16) for _ in range(3)] for _ in range(2)]
    w = [torch.empty((128 * G, d), dtype=dtype, device=DEV) for _ in range(3)]
    layer = cs.Layer(plan, torch.zeros((1, d), device=DEV), torch.zeros((1, G), device=DEV), *w, 1.0)
    h = randn(g, B, d)
    support = torch.tensor([[0, 3], [1, 3], [2, 5]], dtype=torch.int32, device=DEV)
    want = []
    for source in sources:
        for q, out in zip(source, w):
            cs.cs_mx_dequantize(*q, d, out=out)
        torch.cuda.synchronize()
        want.append(cs.cs_ffn_exec(plan, layer, h, support))
        torch.cuda.synchronize()
    assert not torch.equal(*want)
    wrong = torch.zeros((), dtype=torch.int64, device=DEV)
    for i in range(300):
        for q, out in zip(sources[i % 2], w):
            cs.cs_mx_dequantize(*q, d, out=out)
        wrong += (cs.cs_ffn_exec(plan, layer, h, support) != want[i % 2]).sum()
    assert int(wrong) == 0 and plan.device_status() == 0
    plan.close()


@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("d,cols", [(256, 256), (1152, 1151), (4096, 4093)])
def test_quantising_what_the_call_ahead_writes(d, cols, transpose):
    """norm -> quantise (whole chunks, and single elements of an odd width) -> dequantise, nothing in between, for two inputs in turn."""
    B = 33
    g = gen(d)
    plan = cs.Plan(d, 128, 128, 1, 1, 0, "mx4", B, 1e-5)
    xs = [randn(g, B, d) * (1 + i) + i for i in range(2)]
    n = torch.empty((B, d), device=DEV)
    lib, layer_in = plan.lib, [cs.cs_mx_norm(plan, x, want_n=True) for x in xs]
    torch.cuda.synchronize()
    want = []
    for got in layer_in:
        n.copy_(got[3])
        torch.cuda.synchronize()
        codes, scales = cs.cs_mx_quantize(n[:, :cols], transpose=transpose)
        torch.cuda.synchronize()
        want.append((codes, scales.view(torch.uint8), cs.cs_mx_dequantize(codes, scales, B if transpose else cols, torch.float32)))
        torch.cuda.synchronize()
    assert not torch.equal(want[0][0], want[1][0])
    q, s = layer_in[0][1].view(torch.uint8).clone(), layer_in[0][2].view(torch.uint8).clone()
    codes, scales, back = (torch.empty_like(t) for t in want[0])
    stream = torch.cuda.current_stream().cuda_stream
    wrong = torch.zeros((), dtype=torch.int64, device=DEV)
    for i in range(200):
        assert lib.cs_mx_norm(plan.handle, xs[i % 2].data_ptr(), 0, None, 0, None, B, None, n.data_ptr(), q.data_ptr(), s.data_ptr(), stream) == 0
        cs.cs_mx_quantize(n[:, :cols], transpose=transpose, codes=codes, scales=scales)
        cs.cs_mx_dequantize(codes, scales, B if transpose else cols, out=back)
        for a, b in zip((codes, scales, back), want[i % 2]):
            wrong += (a != b).sum()
    assert int(wrong) == 0
    plan.close()


def test_packing_what_the_calls_ahead_write():
    """quantise three matrices, pack, FFN, nothing in between, for two layers in turn in the same place."""
    d, G, k, B = 256, 4, 2, 5
    g = gen(41)
    plan = cs.Plan(d, 128 * G, 128, 1, k, 0, "mx4", B, 1e-5)
    sources = [[randn(g, 128 * G, d) / 16 for _ in range(3)] for _ in range(2)]
    _, q, s, _ = cs.cs_mx_norm(plan, randn(g, B, d))
    support = torch.tensor([[0, 3], [1, 2], [1, 3], [0, 1], [2, 3]], dtype=torch.int32, device=DEV)
    room = [cs.cs_mx_quantize(w, transpose=i == 2) for i, w in enumerate(sources[0])]
    layer = cs.MxLayer(plan, *room)
    matrices = [binding._MxMatrix(c.data_ptr(), e.data_ptr()) for c, e in room]
    stream = torch.cuda.current_stream().cuda_stream

    def run(source, wait):
        for i, (w, (c, e)) in enumerate(zip(source, room)):
            cs.cs_mx_quantize(w, transpose=i == 2, codes=c, scales=e)
        wait()
        assert plan.lib.cs_mx_pack(plan.handle, *(ctypes.byref(m) for m in matrices), *(t.data_ptr() for t in layer.tensors), stream) == 0
        wait()
        return cs.cs_mx_ffn(plan, layer, q, s, support)
    want = [run(source, torch.cuda.synchronize) for source in sources]
    assert not torch.equal(*want)
    torch.cuda.synchronize()
    wrong = torch.zeros((), dtype=torch.int64, device=DEV)
    for i in range(200):
        wrong += (run(sources[i % 2], lambda: None) != want[i % 2]).sum()
    assert int(wrong) == 0 and plan.device_status() == 0
    plan.close()
