"""The operators around the attention call of a video transformer layer, as measurable cases.

Three operators, each as a user's program calls it, and in its plain form in 32-bit torch arithmetic:

  linear   out = act(x W^T + bias) + residual with x and W held in e4m3 codes.  One call quantises the activations (a scale
           per token and 128 inputs), one multiplies (a scale per 128 x 128 tile of the weights).  Weights are quantised once,
           when a model is loaded.
  rope     rotary positions of Q and K: interleaved or half layout, the whole head or a part of it, one position axis or three
           (frame, row, column), frequencies scaled for long contexts, and the inverse rotation, which is the gradient.
  cache    K and V of the tokens computed in this call are quantised into a paged cache (e4m3, or 4-bit codes), and a whole
           sequence is read back into the tensors that attention takes.

Keys of a case: `op`, and
  linear   M tokens, K inputs, N outputs, act ("none", "gelu", "silu"), bias, residual
  rope     B, Hq, Hk, N, d, R (rotated channels), layout ("interleaved", "half"), axes (1 or 3), base, scaling ("none", "linear",
           "ntk", "parts"), factor, length (the trained length), start (first position), inverse, tokens_first ([B, N, H, d])
  cache    do ("write", "read", "step": write, then read), form ("e4m3", "fp4"), B, H, d, page, T (tokens written per sequence),
           N (rows read per sequence), ragged (lengths below N, padding among the written tokens), tokens_first
"""
import math

import torch

own = False


def listed():
    lin = dict(op="linear", act="none", bias=True, residual=False)
    rope = dict(op="rope", B=1, d=128, R=128, axes=1, base=10000.0, scaling="none", factor=1.0, length=4096, start=0, inverse=False)
    cache = dict(op="cache", B=1, d=128, page=64, T=0, N=0, ragged=False, tokens_first=False)
    return [
        # one conditioning vector through a square projection: the smallest product, a call is all that it costs
        dict(lin, name="linear_one_vector", M=1, K=2048, N=2048, act="silu"),
        # the modulation of every layer from the conditioning of a guidance pair: two rows, the weights are the work
        dict(lin, name="linear_modulation_pair", M=2, K=4096, N=24576),
        # a prompt's tokens, sizes that are multiples of nothing
        dict(lin, name="linear_prompt_ragged", M=333, K=2040, N=4104),
        # the FFN's first product of an 8 192-token clip, with its activation
        dict(lin, name="linear_ffn_gelu", M=8192, K=2048, N=8192, act="gelu"),
        # the output projection of a 47 616-token clip of a large model, added to the residual stream; the largest product
        dict(lin, name="linear_out_residual", M=47616, K=4096, N=4096, residual=True),
        # one new token of eight sequences, far into a long context: latency
        dict(rope, name="rope_one_token", B=8, Hq=32, Hk=8, N=1, layout="half", start=131071, base=500000.0, scaling="parts",
             factor=32.0, tokens_first=True),
        # Q and K of the 32 760-token clip, positions on the (frame, row, column) grid
        dict(rope, name="rope_video", Hq=24, Hk=24, N=32760, layout="interleaved", axes=3, tokens_first=False),
        # the gradient of an odd-sized batch, half of each head rotated, grouped keys
        dict(rope, name="rope_gradient_part", B=2, Hq=32, Hk=8, N=8191, R=64, layout="half", scaling="ntk", factor=4.0, inverse=True,
             tokens_first=True),
        # one new token of 64 sequences is written: latency
        dict(cache, name="cache_write_token", do="write", form="e4m3", B=64, H=8, page=16, T=1, N=255, tokens_first=True),
        # a clip's whole K and V are kept for the calls that follow
        dict(cache, name="cache_write_clip", do="write", form="e4m3", H=24, T=32760, N=32760),
        # ... and read back: a guidance pair of the large model
        dict(cache, name="cache_read_pair", do="read", form="e4m3", B=2, H=32, N=47616),
        # a pruned call: half of the tokens are computed again and written, all are read; 4-bit codes, ragged sequences
        dict(cache, name="cache_step_fp4", do="step", form="fp4", B=2, H=16, page=48, T=4001, N=8190, ragged=True, tokens_first=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: single rows to the largest clip, sizes that divide nothing among them, every option."""
    op = rng.choice(("linear", "linear", "rope", "cache"))
    if op == "linear":
        few = rng.random() < 0.4
        while True:
            M = _log_int(rng, 1, 64) if few else _log_int(rng, 65, 47616)
            widths = 512, 768, 1024, 1280, 1536, 2048, 2560, 4096, 5120, 6144, 8192
            K, N = (rng.choice(widths) if rng.random() < 0.5 else 8 + 16 * _log_int(rng, 32, 512) for _ in range(2))
            if M * K * N <= 47616 * 4096 * 4096 and M * N <= 47616 * 4096 and M * K <= 47616 * 4096:
                return dict(op=op, M=M, K=K, N=N, act=rng.choice(("none", "none", "gelu", "silu")), bias=rng.random() < 0.7,
                            residual=rng.random() < 0.4)
    while True:
        B, H, d = rng.choice((1, 1, 2, 3)), _log_int(rng, 1, 32), rng.choice((64, 128, 128))
        tokens_first, N = rng.random() < 0.5, _log_int(rng, 1, 47616)
        if rng.random() < 0.2:
            B, N = _log_int(rng, 1, 64), rng.choice((1, 1, 2, 5))
        if B * H * N * d <= 40_000_000 or rng.random() < 0.3 and B * H * N * d <= 24 * 32760 * 128:
            break
    if op == "rope":
        axes = rng.choice((1, 1, 3))
        return dict(op=op, B=B, Hq=H, Hk=H if rng.random() < 0.5 else max(1, H // 4), N=N, d=d,
                    R=d if rng.random() < 0.5 else 2 * rng.randint(4, d // 2), layout=rng.choice(("interleaved", "half")), axes=axes,
                    base=rng.choice((100.0, 10000.0, 500000.0)), scaling=rng.choice(("none", "linear", "ntk", "parts")),
                    factor=round(rng.uniform(1.0, 32.0), 2), length=rng.choice((2048, 8192)), start=rng.choice((0, 0, rng.randint(1, 1 << 20))),
                    inverse=rng.random() < 0.3, tokens_first=tokens_first)
    do = rng.choice(("write", "read", "step"))
    form = rng.choice(("e4m3", "fp4")) if do != "write" else "e4m3"       # (4-bit codes are seen through the read)
    T = 0 if do == "read" else N if do == "write" else rng.randint(1, N)
    return dict(op=op, do=do, form=form, B=B, H=H, d=d, page=rng.choice((16, 48, 64, 128)), T=T, N=N, ragged=rng.random() < 0.5,
                tokens_first=tokens_first)


def work(case):
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        read = 2 * M * K + N * K + 4 * (-(-N // 128)) * (-(-K // 128)) + 4 * N * case["bias"] + 2 * M * N * case["residual"]
        return {"bytes": float(read + 2 * M * N), "flops": 2.0 * M * K * N}
    if case["op"] == "rope":
        rows = case["B"] * (case["Hq"] + case["Hk"]) * case["N"]
        return {"bytes": 4.0 * rows * case["d"] + 4.0 * case["axes"] * case["B"] * case["N"], "flops": 3.0 * rows * case["R"]}
    d = case["d"]
    held = d + 4 if case["form"] == "e4m3" else d // 2 + d // 16 + 4
    rows = 2 * case["B"] * case["H"] * (case["T"] + (case["N"] if case["do"] != "write" else 0))
    return {"bytes": float(rows * (2 * d + held)), "flops": 2.0 * rows * d}


class State:
    pass


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)


def _heads(gen, B, H, N, d, tokens_first):
    """[B, H, N, d], or the same as a view of [B, N, H, d]."""
    return _randn(gen, B, N, H, d).transpose(1, 2) if tokens_first else _randn(gen, B, H, N, d)


# ---------------------------------------------------------------------------------------------------------- e4m3 and 4-bit codes
def _quotient(a, b):
    """a / b with b a number, divided rather than multiplied by its reciprocal."""
    return a / torch.full((), b, dtype=a.dtype, device=a.device)


def _codes8(x, amax):
    """e4m3 codes (bytes) and scales of fp32 x whose largest magnitudes are amax (broadcast against x)."""
    scale = torch.where(amax == 0, torch.ones_like(amax), _quotient(amax, 448.0))
    return (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8), scale


def _tile_amax(w):
    """Largest magnitude of each 128 x 128 tile of w [N, K]."""
    n, k = -(-w.shape[0] // 128), -(-w.shape[1] // 128)
    padded = torch.zeros(n * 128, k * 128, dtype=torch.float32, device=w.device)
    padded[:w.shape[0], :w.shape[1]] = w.float().abs()
    return padded.view(n, 128, k, 128).amax(dim=(1, 3))


def _spread(scale, n, k):
    """One value per 128 x 128 tile -> [n, k]."""
    return scale.repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]


def _fp4_magnitudes(like):
    return torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=like.dtype, device=like.device)


def _codes4(x):
    """4-bit codes (two per byte, the even channel in the low half), e4m3 scale bytes per 16 channels and fp32 scales per row of fp32 x [.., d]."""
    blocks = x.unflatten(-1, (-1, 16))
    amax = x.abs().amax(-1)
    g = torch.where(amax == 0, torch.ones_like(amax), _quotient(amax, 2688.0))
    sf = (_quotient(blocks.abs().amax(-1), 6.0) / g[..., None]).clamp(max=448.0).to(torch.float8_e4m3fn)
    unit = (sf.float() * g[..., None])[..., None]
    y = torch.where(unit == 0, torch.zeros_like(blocks), blocks / torch.where(unit == 0, torch.ones_like(unit), unit))
    a = y.abs()
    index = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int()
             + (a > 5.0).int())
    code = (index + 8 * (torch.signbit(blocks) & (unit != 0)).int()).flatten(-2).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), sf.view(torch.uint8), g


def _values4(codes, sf, g):
    """What the 4-bit codes stand for, in fp32."""
    low, high = (codes & 15).long(), (codes >> 4).long()
    code = torch.stack((low, high), -1).flatten(-2)
    value = _fp4_magnitudes(g)[code & 7] * torch.where(code >= 8, -1.0, 1.0)
    return (value.unflatten(-1, (-1, 16)) * sf.view(torch.float8_e4m3fn).float()[..., None]).flatten(-2) * g[..., None]


# ---------------------------------------------------------------------------------------------------------- rotary frequencies
def _axis_pairs(case):
    """Pairs of channels that turn with each position axis: as even as they go, the first axis (frames) taking what is left."""
    pairs, axes = case["R"] // 2, case["axes"]
    side = pairs // axes
    return [pairs - side * (axes - 1)] + [side] * (axes - 1)


def _frequencies(case):
    """Radians per position of every pair (64-bit), and the factor on cos and sin."""
    ladders = []
    for pairs in _axis_pairs(case):
        base = case["base"]
        if case["scaling"] == "ntk" and pairs > 1:
            base = base * case["factor"] ** (pairs / (pairs - 1))
        theta = [base ** (-j / pairs) for j in range(pairs)]
        if case["scaling"] == "linear":
            theta = [t / case["factor"] for t in theta]
        if case["scaling"] == "parts":
            turns = [case["length"] * t / (2 * math.pi) for t in theta]
            keep = [min(1.0, max(0.0, (r - 1.0) / 31.0)) for r in turns]
            theta = [t * ((1 - g) / case["factor"] + g) for t, g in zip(theta, keep)]
        ladders += theta
    return ladders, 0.1 * math.log(case["factor"]) + 1.0 if case["scaling"] == "parts" else 1.0


# ---------------------------------------------------------------------------------------------------------- states
def prepare(case, seed):
    s, gen = State(), _generator(seed)
    s.case, s.plan = case, None
    {"linear": _prepare_linear, "rope": _prepare_rope, "cache": _prepare_cache}[case["op"]](s, case, gen)
    return s


def _prepare_linear(s, case, gen):
    M, K, N = case["M"], case["K"], case["N"]
    spread = torch.exp(0.5 * torch.randn(K, generator=gen, device="cuda"))           # channels of different size
    s.x = (torch.randn(M, K, generator=gen, device="cuda") * spread).to(torch.bfloat16)
    w = (torch.randn(N, K, generator=gen, device="cuda") / math.sqrt(K)).to(torch.bfloat16)
    row = -(-K // 16) * 16                                                           # codes: rows of whole 16 bytes
    s.w8 = torch.zeros(N, row, dtype=torch.uint8, device="cuda")
    amax = _tile_amax(w)
    s.w8[:, :K] = _codes8(w.float(), _spread(amax, N, K))[0]
    s.w_scale = _codes8(amax, amax)[1].contiguous()
    s.bias = torch.randn(N, generator=gen, device="cuda") * 0.1 if case["bias"] else None
    s.residual = _randn(gen, M, N) if case["residual"] else None
    s.x8 = torch.empty(M, row, dtype=torch.uint8, device="cuda")
    s.x_scale = torch.empty(-(-K // 128), M, dtype=torch.float32, device="cuda")
    s.out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")


def _prepare_rope(s, case, gen):
    B, N, first = case["B"], case["N"], case["tokens_first"]
    s.q = _heads(gen, B, case["Hq"], N, case["d"], first)
    s.k = _heads(gen, B, case["Hk"], N, case["d"], first)
    if case["axes"] == 1:                                                            # sequences at places of their own
        begin = torch.randint(0, 64, (B, 1), generator=gen, device="cuda") + case["start"]
        s.positions = (begin + torch.arange(N, device="cuda")).to(torch.int32)[None].contiguous()
    else:                                                                            # a grid of frames, the same for the batch
        side = max(1, int(math.sqrt(N / 16)))
        n = torch.arange(N, device="cuda") + side * side * int(torch.randint(0, 8, (1,), generator=gen, device="cuda"))
        s.positions = (torch.stack((n // (side * side), n // side % side, n % side))[:, None] + case["start"]).to(torch.int32).contiguous()
    s.theta, s.factor = _frequencies(case)
    steps = [int(round(t / (2 * math.pi) * 2.0 ** 64)) for t in s.theta]             # fractions of a turn, 64 bits
    s.steps = torch.tensor(steps, dtype=torch.int64, device="cuda")
    s.q_out, s.k_out = torch.empty_like(s.q), torch.empty_like(s.k)


def _prepare_cache(s, case, gen):
    B, H, d, page, T, N = (case[n] for n in ("B", "H", "d", "page", "T", "N"))
    per = -(-N // page)
    pages = B * per + 3
    order = torch.randperm(pages, generator=gen, device="cuda")
    s.table = order[:B * per].view(B, per).to(torch.int32)
    s.lengths = torch.full((B,), N, dtype=torch.int32, device="cuda")
    if case["ragged"]:
        s.lengths = torch.randint(N // 2, N + 1, (B,), generator=gen, device="cuda").to(torch.int32)
    s.cache = []                                                                     # K's arrays, then V's: what was written before
    for _ in range(2):
        x = torch.randn(pages, H, page, d, generator=gen, device="cuda").to(torch.bfloat16).float()
        if case["form"] == "e4m3":
            codes, scale = _codes8(x, x.abs().amax(-1, keepdim=True))
            s.cache.append([codes, scale[..., 0].contiguous()])
        else:
            codes, sf, g = _codes4(x)
            s.cache.append([codes.contiguous(), g.contiguous(), sf.contiguous()])
        del x
    if T:
        s.k, s.v = (_heads(gen, B, H, T, d, case["tokens_first"]) for _ in range(2))
        if T < N:                                                                    # the tokens of this call, in order
            at = torch.stack([torch.randperm(N, generator=gen, device="cuda")[:T].sort().values for _ in range(B)])
        else:
            at = torch.arange(N, device="cuda").expand(B, N)
        slot = torch.gather(s.table.long(), 1, at // page) * page + at % page
        if case["ragged"]:                                                           # padding tokens have no slot
            slot = torch.where(torch.rand(B, T, generator=gen, device="cuda") < 0.05, -1, slot)
        s.slots = slot.to(torch.int32).contiguous()
    if case["do"] != "write":
        s.k_out, s.v_out = (torch.empty_like(_heads(gen, B, H, N, d, case["tokens_first"])) for _ in range(2))


# ---------------------------------------------------------------------------------------------------------- one pass
def run(s):
    return {"linear": _linear, "rope": _rope, "cache": _cache}[s.case["op"]](s)


def _linear(s):
    c = s.case
    if own:
        from paper_2606_23743_b200 import binding as sva
        if s.plan is None:
            s.plan = sva.make_linear(s.x, s.x8, s.x_scale, s.w8, s.w_scale, s.out, c["act"], s.residual)
        sva.quantize_rows_fp8(s.plan, s.x, s.x8, s.x_scale)
        sva.linear_fp8(s.plan, s.x8, s.x_scale, s.w8, s.w_scale, s.out, s.bias, s.residual)
        return s.out
    M, K, N = c["M"], c["K"], c["N"]
    x = torch.zeros(M, -(-K // 128) * 128, dtype=torch.float32, device="cuda")
    x[:, :K] = s.x
    groups = x.view(M, -1, 128)
    codes, scale = _codes8(groups, groups.abs().amax(-1, keepdim=True))
    x = (codes.view(torch.float8_e4m3fn).float() * scale).view(M, -1)[:, :K]
    w = s.w8[:, :K].view(torch.float8_e4m3fn).float() * _spread(s.w_scale, N, K)
    y = x @ w.t()
    if s.bias is not None:
        y = y + s.bias
    if c["act"] == "gelu":
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    elif c["act"] == "silu":
        y = y / (1 + torch.exp(-y))
    if s.residual is not None:
        y = y + s.residual
    return y.to(torch.bfloat16)


def _rotated(x, cos, sin, case):
    R, half = case["R"], case["R"] // 2
    x = x.float()
    if case["layout"] == "half":
        a, b = x[..., :half], x[..., half:R]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((turned, x[..., R:]), -1).to(torch.bfloat16)


def _rope(s):
    c = s.case
    if own:
        from paper_2606_23743_b200 import binding as sva
        if s.plan is None:
            s.plan = sva.make_rope(s.q, s.k, s.q_out, s.k_out, s.positions, c["R"], c["layout"], _axis_pairs(c), s.factor, c["inverse"])
        sva.rope(s.plan, s.q, s.k, s.steps, s.positions, s.q_out, s.k_out)
        return s.q_out, s.k_out
    axis = torch.arange(c["axes"], device="cuda").repeat_interleave(torch.tensor(_axis_pairs(c), device="cuda"), output_size=c["R"] // 2)
    phase = s.positions.long().movedim(0, -1)[..., axis] * s.steps                   # [B or 1, N, pairs], whole turns fall off
    angle = (phase >> 32).float() * (2 * math.pi / 2.0 ** 32)
    cos, sin = torch.cos(angle)[:, None] * s.factor, torch.sin(angle)[:, None] * (-s.factor if c["inverse"] else s.factor)
    return _rotated(s.q, cos, sin, c), _rotated(s.k, cos, sin, c)


def _write(arrays, x, slots, form, page):
    """x [B, H, T, d] into the cache arrays at its tokens' slots; tokens without one are left out."""
    H = x.shape[1]
    slots = slots.flatten().long()
    rows = x.float().transpose(1, 2).flatten(0, 1)[slots >= 0]                       # [tokens, H, d]
    slots = slots[slots >= 0]
    if form == "e4m3":
        codes, scale = _codes8(rows, rows.abs().amax(-1, keepdim=True))
        parts = (codes, scale[..., 0])
    else:
        codes, sf, g = _codes4(rows)
        parts = (codes, g, sf)
    at = slots // page, slots % page
    heads = torch.arange(H, device=x.device)
    [a.index_put_((at[0][:, None], heads[None], at[1][:, None]), p) for a, p in zip(arrays, parts)]


def _read(arrays, table, lengths, form, N):
    taken = [a[table.long()].transpose(1, 2).flatten(2, 3)[:, :, :N] for a in arrays]
    if form == "e4m3":
        x = taken[0].view(torch.float8_e4m3fn).float() * taken[1][..., None]
    else:
        x = _values4(taken[0], taken[2], taken[1])
    there = torch.arange(N, device=x.device)[None] < lengths[:, None]
    return torch.where(there[:, None, :, None], x, torch.zeros_like(x)).to(torch.bfloat16)


def _cache(s):
    c = s.case
    k, v = s.cache
    if own:
        from paper_2606_23743_b200 import binding as sva
        if s.plan is None:
            s.plan = sva.make_kv_cache(k, v, c["form"])
        if c["do"] != "read":
            sva.kv_cache_write(s.plan, s.k, s.v, s.slots)
        if c["do"] != "write":
            sva.kv_cache_read(s.plan, s.table, s.lengths, s.k_out, s.v_out)
            return s.k_out, s.v_out
    else:
        if c["do"] != "read":
            _write(k, s.k, s.slots, c["form"], c["page"])
            _write(v, s.v, s.slots, c["form"], c["page"])
        if c["do"] != "write":
            return _read(k, s.table, s.lengths, c["form"], c["N"]), _read(v, s.table, s.lengths, c["form"], c["N"])
    return k[0].view(torch.float8_e4m3fn), k[1], v[0].view(torch.float8_e4m3fn), v[1]


# ---------------------------------------------------------------------------------------------------------- in 64 bits
def _nearest(y, least, mantissa, top):
    """y rounded to the nearest number of a small floating-point format (ties to even): exponents from `least`, so many bits."""
    exponent = torch.frexp(y)[1].clamp(min=least + 1) - 1
    unit = torch.ldexp(torch.ones_like(y), exponent - mantissa)
    return (torch.round(y / unit) * unit).clamp(-top, top)


def _as_fp32(y):
    return y.to(torch.float32).to(torch.float64)


def _exact8(x):
    """(codes' values, scale) of the rows of x, in 64 bits: the scale and the quotient are fp32 numbers by definition."""
    top = x.abs().amax(-1, keepdim=True)
    scale = torch.where(top > 0, _as_fp32(top / 448.0), 1.0)
    return _nearest(_as_fp32(x / scale), -6, 3, 448.0), scale


def _exact4(x):
    """What x is after its way through 4 bits, in 64 bits."""
    shape, top = x.shape, x.abs().amax(-1, keepdim=True)
    g = torch.where(top > 0, _as_fp32(top / 2688.0), 1.0)
    x = x.reshape(*shape[:-1], shape[-1] // 16, 16)
    g = g[..., None]
    sf = _nearest(_as_fp32(_as_fp32(x.abs().amax(-1, keepdim=True) / 6.0) / g), -6, 3, 448.0)
    unit = _as_fp32(sf * g)
    code = torch.where(unit > 0, _nearest(_as_fp32(x / torch.where(unit > 0, unit, 1.0)), 0, 1, 6.0), 0.0)
    return (code * sf * g).reshape(shape)


def exact(case, seed):
    s = prepare(case, seed)
    return {"linear": _exact_linear, "rope": _exact_rope, "cache": _exact_cache}[case["op"]](s, case)


def _exact_linear(s, case):
    M, K, N = case["M"], case["K"], case["N"]
    y = torch.zeros(M, N, dtype=torch.float64, device="cuda")
    w = s.w8.view(torch.float8_e4m3fn).double()
    at = torch.arange(N, device="cuda") // 128
    for g in range(-(-K // 128)):
        lo, hi = 128 * g, min(K, 128 * g + 128)
        code, scale = _exact8(s.x[:, lo:hi].double())
        y.addmm_(code * scale, (w[:, lo:hi] * s.w_scale[at, g].double()[:, None]).t())
    if case["bias"]:
        y += s.bias.double()
    if case["act"] == "gelu":
        y = 0.5 * y * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (y + 0.044715 * y ** 3)))
    elif case["act"] == "silu":
        y = y * torch.sigmoid(y)
    return y + s.residual.double() if case["residual"] else y


def _exact_rope(s, case):
    half, outs = case["R"] // 2, []
    theta = torch.tensor(s.theta, dtype=torch.float64, device="cuda")
    pos = torch.cat([s.positions[a].double()[..., None].expand(-1, -1, p) for a, p in enumerate(_axis_pairs(case))], -1)
    angle = (pos * theta)[:, None] * (-1.0 if case["inverse"] else 1.0)
    turn = torch.polar(torch.full_like(angle, s.factor), angle)                      # a rotation is a complex product
    for x in (s.q, s.k):
        y = x.double()
        at = torch.arange(case["R"], device="cuda")
        first, second = (at[:half], at[half:]) if case["layout"] == "half" else (at[0::2], at[1::2])
        z = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        outs.append(y)
    return tuple(outs)


def _exact_cache(s, case):
    B, H, d, page, N = case["B"], case["H"], case["d"], case["page"], case["N"]
    outs = []
    for arrays, x in zip(s.cache, (s.k, s.v) if case["T"] else (None, None)):
        codes = arrays[0]
        if case["form"] == "e4m3":
            value, scale = codes.view(torch.float8_e4m3fn).double(), arrays[1].double()
            if x is not None:
                new, new_scale = _exact8(x.double())
                for b in range(B):
                    keep = s.slots[b] >= 0
                    to = s.slots[b][keep].long()
                    value[to // page, :, to % page] = new[b][:, keep].transpose(0, 1)
                    scale[to // page, :, to % page] = new_scale[b][:, keep, 0].t()
            if case["do"] == "write":
                outs += [value, scale]
                continue
            held = value * scale[..., None]
        else:
            pairs = torch.stack((codes % 16, codes // 16), -1).reshape(*codes.shape[:-1], d).double()
            size, sign = pairs % 8, torch.where(pairs >= 8, -1.0, 1.0)
            size = torch.where(size < 2, size / 2, (1 + size % 2 / 2) * 2.0 ** (torch.floor(size / 2) - 1))
            factors = arrays[2].view(torch.float8_e4m3fn).double() * arrays[1].double()[..., None]
            held = sign * size * factors.repeat_interleave(16, -1)
            if x is not None:
                new = _exact4(x.double())
                for b in range(B):
                    keep = s.slots[b] >= 0
                    to = s.slots[b][keep].long()
                    held[to // page, :, to % page] = new[b][:, keep].transpose(0, 1)
        y = torch.zeros(B, H, N, d, dtype=torch.float64, device="cuda")
        for b in range(B):
            n = torch.arange(int(s.lengths[b]), device="cuda")
            y[b][:, n] = held[s.table[b].long()[n // page], :, n % page].transpose(0, 1)
        outs.append(y)
    return tuple(outs)
