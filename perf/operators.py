"""Cases for the microscaled low-precision operators: 4-bit weights, the 8-bit norm in front of them, and the FFN between the two.

What a case stands for is its "kind":
  quant   weights to blocks of 32 four-bit elements with a power-of-two scale each, and back to the type they came in: what a
          program does when it loads a layer (and when it checks what the quantisation costs)
  norm    the previous block's output added to the residual stream, RMSNorm, and the result in 8-bit blocks
  ffn     the SwiGLU FFN of B tokens over the groups of their supports, 8-bit activations and 4-bit weights: decode
          batches whose tokens have supports of their own, and prompts that share one

Block format: 32 consecutive elements share a scale 2^e, e the smallest integer (not below -127) for which the block's largest magnitude is at most
M 2^e, M = 6 for 4-bit (e2m1) and 448 for 8-bit (e4m3) elements; elements are rounded to nearest, ties to even.
Shapes are those of gen/workloads.py and around them.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 128
EPS = 1e-5
_7B = dict(d=4096, G=86, k=22)
_8B = dict(d=4096, G=112, k=28)
_13B = dict(d=5120, G=108)
_MOST_FLOPS = 6 * 2048 * 27 * GROUP * 5120


def listed():
    return [
        # a toy layer's weights: launches and latency only
        dict(name="quant_tiny_f32", kind="quant", rows=1024, cols=256, dtype="f32", transpose=False),
        # one projection of a 7B layer, as loading a model does 3 times per layer
        dict(name="quant_7b_gate", kind="quant", rows=11008, cols=4096, dtype="bf16", transpose=False),
        # the down projection, which the framework stores transposed: blocks run down the columns
        dict(name="quant_7b_down", kind="quant", rows=11008, cols=4096, dtype="bf16", transpose=True),
        # decoding one sequence: latency
        dict(name="norm_7b_b1", kind="norm", B=1, d=4096, dtype="f32", delta=True, want_n=True),
        # a serving batch, with the f32 rows that the sketch reads
        dict(name="norm_7b_b64", kind="norm", B=64, d=4096, dtype="f32", delta=True, want_n=True),
        # a prompt
        dict(name="norm_13b_n2048", kind="norm", B=2048, d=5120, dtype="bf16", delta=True, want_n=False),
        # decoding one sequence
        dict(name="ffn_7b_b1", kind="ffn", B=1, shared=False, **_7B),
        # a few sequences, nearly disjoint supports
        dict(name="ffn_7b_b3", kind="ffn", B=3, shared=False, **_7B),
        # a serving batch
        dict(name="ffn_7b_b64", kind="ffn", B=64, shared=False, **_7B),
        # an odd batch of another layer
        dict(name="ffn_8b_b200", kind="ffn", B=200, shared=False, **_8B),
        # a ragged prompt at 10 % of the groups, and the 2048-token one at 25 %
        dict(name="ffn_13b_n777", kind="ffn", B=777, k=11, shared=True, **_13B),
        dict(name="ffn_13b_n2048", kind="ffn", B=2048, k=27, shared=True, **_13B),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(["quant", "norm", "ffn"], [2, 2, 4])[0]
    if kind == "quant":
        cols = _log_int(rng, 1, 8192)
        rows = _log_int(rng, 1, min(16384, 11008 * 4096 // cols))
        return dict(kind=kind, rows=rows, cols=cols, dtype=rng.choice(["f32", "bf16"]), transpose=rng.random() < 0.5)
    if kind == "norm":
        return dict(kind=kind, B=_log_int(rng, 1, 2048), d=GROUP * rng.randint(2, 40), dtype=rng.choice(["f32", "bf16"]),
                    delta=rng.random() < 0.75, want_n=rng.random() < 0.5)
    d = GROUP * rng.randint(2, 40)
    G = rng.randint(2, min(128, 112 * 4096 // d))
    k = max(1, min(G, int(round(G * rng.uniform(0.05, 0.6)))))
    shared = rng.random() < 0.4
    B = _log_int(rng, 16, 2048) if shared else _log_int(rng, 1, 300)
    B = max(1, min(B, _MOST_FLOPS // (6 * k * GROUP * d)))
    return dict(kind=kind, B=B, d=d, G=G, k=k, shared=shared)


# ---- inputs ----------------------------------------------------------------------------------------

_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_TYPES = dict(f32=torch.float32, bf16=torch.bfloat16)


def _e8m0(e):
    return (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _pow2(e):
    """2^e in f32, e from -127 to 127."""
    return _e8m0(e).float()


def _exponent(amax, top_mantissa, top_exponent):
    """The block's exponent: amax = m 2^p with m in [0.5, 1), M = top_mantissa 2^top_exponent."""
    m, p = torch.frexp(amax)
    e = p - top_exponent + (m > top_mantissa).to(p.dtype)
    return torch.where(amax > 0, e, torch.full_like(e, -127)).clamp_min(-127)


def _to_mx4(w):
    """f32 [rows, cols], cols a multiple of 32 -> (e2m1 values as f32 [rows, cols / 32, 32], exponents [rows, cols / 32])."""
    b = w.reshape(w.shape[0], -1, 32)
    e = _exponent(b.abs().amax(-1), 0.75, 3)
    x = b * _pow2(-e).unsqueeze(-1)
    a = x.abs()
    a = torch.where(a < 2, torch.round(a * 2) / 2, torch.where(a < 4, torch.round(a), torch.round(a / 2) * 2))
    return torch.copysign(a, x), e


def _to_mx8(n):
    """f32 [rows, cols], cols a multiple of 32 -> (e4m3 [rows, cols], exponents [rows, cols / 32])."""
    b = n.reshape(n.shape[0], -1, 32)
    e = _exponent(b.abs().amax(-1), 0.875, 9)
    return (b * _pow2(-e).unsqueeze(-1)).to(torch.float8_e4m3fn).reshape(n.shape), e


def _pack(v):
    """e2m1 values [rows, blocks, 32] -> two codes to a byte [rows, 16 blocks], the even element in the low half."""
    code = torch.bucketize(v.abs(), torch.tensor(_E2M1, device=v.device)).to(torch.uint8) | (torch.signbit(v).to(torch.uint8) << 3)
    code = code.reshape(v.shape[0], -1)
    return code[:, 0::2] | (code[:, 1::2] << 4)


def _tiles(e):
    """Exponents [rows, blocks] as e8m0 scales in the tensor cores' tile order: [rows / 128, blocks / 4] tiles of [32][4][4], byte
    [r % 32][r / 32][b % 4] of a tile for row r, block b; 2^-127 behind the last row and block."""
    R, C = -(-e.shape[0] // 128), -(-e.shape[1] // 4)
    p = torch.full((128 * R, 4 * C), -127, dtype=e.dtype, device=e.device)
    p[:e.shape[0], :e.shape[1]] = e
    return _e8m0(p.reshape(R, 4, 32, C, 4).permute(0, 3, 2, 1, 4).contiguous())


def _untiles(s, rows):
    """The scales of _tiles as f32 [rows, blocks]."""
    R, C = s.shape[:2]
    return s.view(torch.uint8).permute(0, 3, 2, 1, 4).reshape(128 * R, 4 * C)[:rows].view(torch.float8_e8m0fnu).float()


def _weights(g, rows, cols, std, dev):
    v, e = _to_mx4(torch.randn((rows, cols), generator=g, device=dev) * std)
    return _pack(v), _e8m0(e)


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    g = torch.Generator(device=dev)
    g.manual_seed(1_000_003 * int(seed) + 17)
    state = dict(case)
    if case["kind"] == "quant":
        std = 1.0 / math.sqrt(case["rows"] if case["transpose"] else case["cols"])
        w = torch.randn((case["rows"], case["cols"]), generator=g, device=dev) * std
        state["w"] = w.to(_TYPES[case["dtype"]])
    elif case["kind"] == "norm":
        B, d = case["B"], case["d"]
        # a residual stream: rows of different size, a few channels far above the others
        size = torch.exp(torch.randn((B, 1), generator=g, device=dev))
        hot = 1 + 30 * (torch.rand((1, d), generator=g, device=dev) < 0.004)
        state["x"] = (torch.randn((B, d), generator=g, device=dev) * size * hot).to(_TYPES[case["dtype"]])
        state["add"] = (torch.randn((B, d), generator=g, device=dev) * 0.3).bfloat16() if case["delta"] else None
        state["gamma"] = 1 + 0.1 * torch.randn((d,), generator=g, device=dev)
    else:
        B, d, G, k = case["B"], case["d"], case["G"], case["k"]
        d_ff = G * GROUP
        state["gate"], state["up"] = (_weights(g, d_ff, d, 1 / math.sqrt(d), dev) for _ in range(2))
        state["down"] = _weights(g, d, d_ff, 1 / math.sqrt(d_ff), dev)
        q, e = _to_mx8(torch.randn((B, d), generator=g, device=dev))
        state["q"], state["s"] = q, _tiles(e)
        draws = torch.rand((1 if case["shared"] else B, G), generator=g, device=dev)
        support = draws.topk(k, dim=1).indices.sort(dim=1).values.to(torch.int32)
        state["support"] = support[0].contiguous() if case["shared"] else support
    if own:
        import paper_2604_14156_b200 as cs
        state["cs"] = cs
        if case["kind"] == "norm":
            state["plan"] = cs.Plan(case["d"], GROUP, GROUP, 1, 1, 0, "mx4", case["B"], EPS)
        elif case["kind"] == "ffn":
            state["plan"] = cs.Plan(d, d_ff, GROUP, 1, k, 0, "mx4", B, EPS)
            state["layer"] = cs.MxLayer(state["plan"], state["gate"], state["up"], state["down"])
    return state


# ---- the operators ---------------------------------------------------------------------------------

def _values4(codes, scales):
    """What 4-bit codes and their scales stand for, f32 [rows, 32 blocks]."""
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)
    v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), -1)
    return (v.reshape(codes.shape[0], -1, 32) * scales.float().unsqueeze(-1)).reshape(codes.shape[0], -1)


def _quant(state):
    w = state["w"].float()
    w = w.t() if state["transpose"] else w
    cols = w.shape[1]
    v, e = _to_mx4(torch.nn.functional.pad(w, (0, -cols % 32)))
    back = (v * _pow2(e).unsqueeze(-1)).reshape(w.shape[0], -1)[:, :cols]
    return dict(values=back.to(state["w"].dtype).contiguous(), scales=_e8m0(e))


def _norm(state):
    h = state["x"] if state["add"] is None else (state["x"].float() + state["add"].float()).to(state["x"].dtype)
    f = h.float()
    n = f / torch.sqrt(f.square().mean(1, keepdim=True) + EPS) * state["gamma"]
    q, e = _to_mx8(n)
    got = dict(h=h, q=q, s=_tiles(e))
    return dict(got, n=n) if state["want_n"] else got


def _ffn(state):
    B, d, G = state["B"], state["d"], state["G"]
    x = state["q"].float().reshape(B, -1, 32) * _untiles(state["s"], B).unsqueeze(-1)
    x = x.reshape(B, d)
    few = state["shared"] or B == 1      # one support: its groups alone
    support = state["support"].reshape(-1, state["k"]).long()
    pick = (lambda t: t.reshape((G, GROUP) + t.shape[1:])[support[0]].flatten(0, 1)) if few else (lambda t: t)
    gate = x @ _values4(pick(state["gate"][0]), pick(state["gate"][1].view(torch.uint8)).view(torch.float8_e8m0fnu)).t()
    up = x @ _values4(pick(state["up"][0]), pick(state["up"][1].view(torch.uint8)).view(torch.float8_e8m0fnu)).t()
    a = gate * torch.sigmoid(gate) * up
    if not few:
        member = torch.zeros((B, G), device=x.device).scatter_(1, support, 1.0)
        a = a * member.repeat_interleave(GROUP, dim=1)
    q, e = _to_mx8(a)
    a = (q.float().reshape(B, -1, 32) * _pow2(e).unsqueeze(-1)).reshape(a.shape)
    codes, scales = state["down"][0], state["down"][1].view(torch.uint8)
    if few:
        codes = codes.reshape(d, G, GROUP // 2)[:, support[0]].flatten(1)
        scales = scales.reshape(d, G, GROUP // 32)[:, support[0]].flatten(1)
    return dict(out=(a @ _values4(codes, scales.view(torch.float8_e8m0fnu)).t()).bfloat16())


def _own(state):
    cs = state["cs"]
    if state["kind"] == "quant":
        codes, scales = cs.cs_mx_quantize(state["w"], transpose=state["transpose"])
        cols = state["w"].shape[0 if state["transpose"] else 1]
        return dict(values=cs.cs_mx_dequantize(codes, scales, cols, state["w"].dtype), scales=scales)
    if state["kind"] == "norm":
        h, q, s, n = cs.cs_mx_norm(state["plan"], state["x"], state["gamma"], delta=state["add"], want_n=state["want_n"])
        got = dict(h=h, q=q, s=s)
        return dict(got, n=n) if state["want_n"] else got
    ffn = cs.cs_mx_ffn_shared if state["shared"] else cs.cs_mx_ffn
    return dict(out=ffn(state["plan"], state["layer"], state["q"], state["s"], state["support"]))


def run(state):
    if own:
        return _own(state)
    return dict(quant=_quant, norm=_norm, ffn=_ffn)[state["kind"]](state)


def work(case):
    if case["kind"] == "quant":
        n = case["rows"] * case["cols"]
        blocks = -(-case["rows"] // 32) * case["cols"] if case["transpose"] else case["rows"] * -(-case["cols"] // 32)
        size = 4 if case["dtype"] == "f32" else 2
        # there: elements read, codes and scales written; back: the reverse
        return dict(bytes=2 * (n * size + 17 * blocks), flops=4 * n)
    if case["kind"] == "norm":
        n = case["B"] * case["d"]
        size = 4 if case["dtype"] == "f32" else 2
        return dict(bytes=n * (size + (2 + size if case["delta"] else 0) + 1 + (4 if case["want_n"] else 0)) + n // 32 + 4 * case["d"], flops=6 * n)
    B, d, G, k = case["B"], case["d"], case["G"], case["k"]
    union = k if case["shared"] else G * (1 - (1 - k / G) ** B)     # groups in use, on average
    weights = union * 3 * GROUP * d * 17 / 32
    return dict(bytes=weights + B * d * 33 / 32 + 2 * B * d + 4 * k * (1 if case["shared"] else B), flops=6 * B * k * GROUP * d)


# ---- the same from the definitions, in 64 bits -------------------------------------------------------

def _two_to(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _grid(amax, largest):
    """2^e in f64, e the smallest integer >= -127 with amax <= largest 2^e; 2^-127 for amax = 0."""
    e = torch.ceil(torch.log2(torch.clamp(amax, min=1e-60) / largest))
    e = torch.where(amax > largest * _two_to(e), e + 1, e)          # the logarithm's own rounding
    e = torch.where(amax <= largest * _two_to(e - 1), e - 1, e)
    return _two_to(e.clamp_min(-127.0))


def _nearest(x, bits, smallest):
    """x in f64 to `bits` bits after the leading one, the spacing never below `smallest`, ties to even."""
    m, p = torch.frexp(x.abs().clamp_min(1e-60))
    step = _two_to(p - 1 - bits).clamp_min(smallest)
    return torch.round(x / step) * step


def _round8(n):
    b = n.reshape(n.shape[0], -1, 32)
    s = _grid(b.abs().amax(-1, keepdim=True), 448.0)
    return _nearest(b / s, 3, 2.0 ** -9), s


def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    if case["kind"] == "quant":
        w = state["w"].double()
        w = w.t().contiguous() if case["transpose"] else w
        rows, cols = w.shape
        blocks = -(-cols // 32)
        full = torch.zeros((rows, 32 * blocks), dtype=torch.float64, device=w.device)
        full[:, :cols] = w
        b = full.reshape(rows, blocks, 32)
        s = _grid(b.abs().amax(-1, keepdim=True), 6.0)
        return dict(values=(_nearest(b / s, 1, 0.5) * s).reshape(rows, -1)[:, :cols].contiguous(), scales=s.squeeze(-1))
    if case["kind"] == "norm":
        h = state["x"].double()
        if state["add"] is not None:
            h = (h + state["add"].double()).to(state["x"].dtype).double()
        n = h / torch.sqrt((h * h).sum(1, keepdim=True) / case["d"] + EPS) * state["gamma"].double()
        q, s = _round8(n)
        R, C = -(-case["B"] // 128), -(-case["d"] // 128)
        tiles = torch.full((R, C, 32, 4, 4), 2.0 ** -127, dtype=torch.float64, device=n.device)
        r, b = torch.arange(case["B"], device=n.device)[:, None], torch.arange(case["d"] // 32, device=n.device)[None, :]
        tiles[r // 128, b // 4, r % 32, r % 128 // 32, b % 4] = s.squeeze(-1)
        got = dict(h=h, q=q.reshape(n.shape), s=tiles)
        return dict(got, n=n) if case["want_n"] else got
    B, d, G, k = case["B"], case["d"], case["G"], case["k"]
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), dtype=torch.float64, device=state["q"].device)

    def values(w, group, down):
        codes, scales = w[0], w[1].double()
        if down:
            codes, scales = codes[:, 64 * group:64 * group + 64], scales[:, 4 * group:4 * group + 4]
        else:
            codes, scales = codes[128 * group:128 * group + 128], scales[128 * group:128 * group + 128]
        both = torch.stack((codes % 16, codes // 16), -1).reshape(codes.shape[0], -1).long()
        return table[both] * scales.repeat_interleave(32, dim=1)

    r, b = torch.arange(B, device=table.device)[:, None], torch.arange(d // 32, device=table.device)[None, :]
    scale = state["s"].double()[r // 128, b // 4, r % 32, r % 128 // 32, b % 4]
    x = state["q"].double() * scale.repeat_interleave(32, dim=1)
    support = state["support"].reshape(-1, k)
    out = torch.zeros((B, d), dtype=torch.float64, device=x.device)
    for group in torch.unique(support).tolist():
        rows = slice(None) if case["shared"] else (support == group).any(1)
        g, u = x[rows] @ values(state["gate"], group, False).t(), x[rows] @ values(state["up"], group, False).t()
        q, s = _round8(g / (1 + torch.exp(-g)) * u)
        out[rows] += (q * s).reshape(-1, GROUP) @ values(state["down"], group, True).t()
    return dict(out=out)
