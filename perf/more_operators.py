"""Microscaled 4-bit weights and the experts' tokens: the operators whose speed is tracked here.

A case is a dict of plain values:

  call    "quantize": one spp_mx4_quantize and the spp_mx4_load that reads the rows back
          "matmul": one spp_mx4_matmul
          "experts": one spp_mx4_experts, the routed FFN of a layer whose experts are resident in 4 bits
          "route": spp_expert_sort, spp_expert_gather and spp_expert_combine; with grad also
          spp_expert_combine_grad and the gather's gradient (spp_expert_combine without weights)
  rows, cols         rows and their elements (quantize)
  M, N, K, groups    rows of x, rows of a group's weights, the elements they share, groups (matmul); with
                     more than one group, M rows fall to them unevenly
  T, n, K, D, I      tokens, routed experts, experts a token, hidden size, SwiGLU intermediate size (experts, route)
  act     "bf16": the products take x in bf16; "mx4": x (and the SwiGLU's result) in 4 bits as well
  dtype   "bf16" or "f32": rows (quantize, route), the output (matmul; experts give bf16)

4 bits: an element is its code's value (a sign and 0, 0.5, 1, 1.5, 2, 3, 4 or 6, two codes to a byte, the even
element low) times 2^(scale byte - 127), one scale byte for 32 elements of a row.
"""
import math

import torch

own = False

DEV = "cuda:0"
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------------- cases

def _named(c, name):
    return dict(c, name=name) if name else c


def _quant(rows, cols, dtype, name=None):
    return _named(dict(call="quantize", rows=rows, cols=cols, dtype=dtype), name)


def _matmul(M, N, K, act, dtype, groups=1, name=None):
    return _named(dict(call="matmul", M=M, N=N, K=K, act=act, dtype=dtype, groups=groups), name)


def _experts(T, n, K, D, I, act, name=None):
    return _named(dict(call="experts", T=T, n=n, K=K, D=D, I=I, act=act, dtype="bf16"), name)


def _route(T, n, K, D, dtype, grad, name=None):
    return _named(dict(call="route", T=T, n=n, K=K, D=D, dtype=dtype, grad=grad), name)


def listed():
    return [
        # one token's hidden state into 4 bits and back (latency)
        _quant(1, 2048, "bf16", name="quantize_b1"),
        # gate and up rows of 64 experts, as weights are brought into the format
        _quant(98304, 2048, "bf16", name="quantize_weights"),
        # queries, keys and values of one token (latency: weights streamed once)
        _matmul(1, 5120, 2048, "bf16", "bf16", name="matmul_b1"),
        # a few uneven groups, fp32 results, sizes off every tile
        _matmul(333, 1000, 1312, "bf16", "f32", groups=5, name="matmul_groups_odd"),
        # a long prompt with both sides in 4 bits
        _matmul(8192, 5120, 2048, "mx4", "bf16", name="matmul_prompt_mx4"),
        # one token through its 8 of 128 experts
        _experts(1, 128, 8, 2048, 768, "bf16", name="experts_b1"),
        # a decode batch of 64 sequences: nearly every expert, a few tokens each
        _experts(64, 128, 8, 2048, 768, "bf16", name="experts_b64"),
        # a chunk of a prompt through the smaller model's experts, exact activations
        _experts(1024, 64, 6, 1280, 896, "bf16", name="experts_chunk"),
        # a long prompt, both sides of every product in 4 bits
        _experts(4096, 128, 8, 2048, 768, "mx4", name="experts_prompt_mx4"),
        # the tokens of a decode batch to their experts and back
        _route(64, 128, 8, 2048, "bf16", False, name="route_b64"),
        # a training batch's tokens, there and back with every gradient
        _route(8192, 128, 8, 2048, "bf16", True, name="route_train"),
        # fp32 with gradients, an odd count
        _route(1237, 64, 6, 1280, "f32", True, name="route_f32_odd"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of these ranges, no costlier than the largest listed one."""
    most = [max(work(c)[k] for c in listed()) for k in ("bytes", "flops")]
    while True:
        c = _draw(rng)
        w = work(c)
        if w["bytes"] <= most[0] and w["flops"] <= most[1]:
            return c


def _draw(rng):
    call = rng.choice(["quantize", "matmul", "matmul", "matmul", "experts", "experts", "experts", "route", "route"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    act = rng.choice(["bf16", "mx4"])
    if call == "quantize":
        return _quant(_log(rng, 1, 100000), 32 * _log(rng, 1, 128), dtype)
    if call == "matmul":
        groups = rng.choice([1, 1, _log(rng, 2, 64)])
        return _matmul(_log(rng, 1, 8192), _log(rng, 16, 6000 if groups == 1 else 2000), 32 * _log(rng, 1, 160), act, dtype,
                       groups)
    n, K = rng.choice([8, 24, 40, 64, 96, 128]), rng.randint(1, 8)
    if call == "experts":
        return _experts(_log(rng, 1, 4096), n, K, 32 * _log(rng, 8, 80), 32 * _log(rng, 4, 36), act)
    return _route(_log(rng, 1, 8192), n, K, 8 * _log(rng, 4, 320), dtype, rng.random() < 0.6)


# --------------------------------------------------------------------- inputs

def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEV).manual_seed(seed)
    call = c["call"]
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
    s = dict(case=c, dt=dt)

    def normal(*shape, dtype=dt):
        return torch.empty(shape, device=DEV).normal_(generator=g).to(dtype)

    if call == "quantize":
        R, C = c["rows"], c["cols"]
        s["x"] = normal(R, C)
        s["x"][:, ::61] *= 20.0  # a few channels are much larger than the rest
        s["codes"] = torch.empty((R, C // 2), dtype=torch.uint8, device=DEV)
        s["scales"] = torch.empty((R, C // 32), dtype=torch.uint8, device=DEV)
        s["out"] = torch.empty((R, C), dtype=dt, device=DEV)
    elif call == "matmul":
        M, N, K, G = c["M"], c["N"], c["K"], c["groups"]
        s["w"] = _weights(G * N, K, g)
        share = torch.rand(G, generator=g, device=DEV) ** 2
        ends = torch.cumsum(share / share.sum(), 0)[:-1].mul(M).round().clamp(0, M)
        s["start"] = torch.cat([ends.new_zeros(1), ends, ends.new_full((1,), M)]).to(torch.int32)
        x = normal(M, K, dtype=torch.bfloat16)
        if c["act"] == "mx4":
            s["xq"] = _quantise(x.float())
        else:
            s["x"] = x
        s["out"] = torch.empty((M, N), dtype=dt, device=DEV)
    else:
        T, n, K, D = c["T"], c["n"], c["K"], c["D"]
        # some experts are more popular than others; a token's are all different
        logits = torch.randn((T, n), generator=g, device=DEV) * 1.5 + torch.randn(n, generator=g, device=DEV) * 0.5
        top, ids = logits.topk(K, dim=1)
        s["topk"] = ids.to(torch.int32).contiguous()
        s["gates"] = torch.softmax(top, dim=1).contiguous()
        s["x"] = normal(T, D)
        s["out"] = torch.empty((T, D), dtype=dt, device=DEV)
        if call == "experts":
            s["gate_up"] = _weights(n * 2 * c["I"], D, g)
            s["down"] = _weights(n * D, c["I"], g)
        else:
            P = T * K
            s["y"] = normal(P, D)
            s["start"] = torch.empty(n + 1, dtype=torch.int32, device=DEV)
            s["pair"], s["place"] = (torch.empty(P, dtype=torch.int32, device=DEV) for _ in range(2))
            s["rows"] = torch.empty((P, D), dtype=dt, device=DEV)
            if c["grad"]:
                s["d_out"], s["d_in"] = normal(T, D), normal(P, D)
                s["d_y"] = torch.empty((P, D), dtype=dt, device=DEV)
                s["d_gates"] = torch.empty((T, K), device=DEV)
                s["d_x"] = torch.empty((T, D), dtype=dt, device=DEV)
    if own:  # a program keeps its weights' descriptions, and one workspace for its calls
        _plan(s)
    return s


def _weights(rows, cols, g):
    """Codes and scales of a normal matrix, as trained weights are stored (a part at a time: its fp32 form is large)."""
    std, part = 1.0 / math.sqrt(cols), max(1, (1 << 26) // cols)
    done = [_quantise(torch.empty((min(part, rows - at), cols), device=DEV).normal_(0.0, std, generator=g))
            for at in range(0, rows, part)]
    return torch.cat([q for q, _ in done]), torch.cat([e for _, e in done])


# ------------------------------------------------------------ the plain forms

def _quantise(x):
    """Codes (two to a byte) and scale bytes of x [rows, cols]: blocks of 32, the smallest power of two with no element
    beyond 7 of it."""
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    finite = torch.isfinite(top)
    part, e = torch.frexp(torch.where(finite, top, 1.0))
    e = torch.where(part <= 0.875, e - 3, e - 2)
    e = torch.where(top > 0, e, -125).clamp(-125, 125)
    a = torch.ldexp(x.abs(), -e)
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
            + 8 * torch.signbit(x).to(torch.uint8))
    code = torch.where(finite, code, 0).flatten(-2).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.where(finite, e + 127, 255).squeeze(-1).to(torch.uint8)


def _values(code, scale):
    """fp32 values of codes [rows, cols/2] with scale bytes [rows, cols/32]."""
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=code.device)
    pair = torch.stack([code & 15, code >> 4], dim=-1).flatten(-2)
    unit = torch.where(scale == 255, float("nan"), torch.ldexp(torch.ones((), device=code.device), scale.int() - 127))
    return (table[pair.int()].unflatten(-1, (-1, 32)) * unit[..., None]).flatten(-2)


def _grouped(x, start, w):
    """Rows start[g] .. start[g+1] - 1 of x times the transpose of w[g], for every g: groups padded to the longest one."""
    start = start.long()
    count = start[1:] - start[:-1]
    j = torch.arange(int(count.max()), device=DEV)
    row = (start[:-1, None] + j).clamp(max=x.shape[0] - 1)
    y = torch.bmm(x[row], w.transpose(1, 2))
    i = torch.arange(x.shape[0], device=DEV)
    group = torch.searchsorted(start[1:].contiguous(), i, right=True)
    return y[group, i - start[group]]


def _order(topk, n):
    """start [n+1], and the pairs' stable order by expert with its inverse."""
    ids = topk.flatten().long()
    pair = torch.argsort(ids, stable=True)
    place = torch.empty_like(pair)
    place[pair] = torch.arange(pair.numel(), device=DEV)
    start = torch.zeros(n + 1, dtype=torch.long, device=DEV)
    start[1:] = torch.cumsum((ids[:, None] == torch.arange(n, device=DEV)).long().sum(0), 0)
    return start, pair, place


def _plain(s):
    c = s["case"]
    call = c["call"]
    if call == "quantize":
        return _values(*_quantise(s["x"])).to(s["dt"])
    if call == "matmul":
        x = _values(*s["xq"]) if c["act"] == "mx4" else s["x"].float()
        w = _values(*s["w"])
        y = x @ w.T if c["groups"] == 1 else _grouped(x, s["start"], w.unflatten(0, (c["groups"], -1)))
        return y.to(s["dt"])
    T, n, K, D = c["T"], c["n"], c["K"], c["D"]
    if call == "experts":
        used = torch.unique(s["topk"]).long()  # the experts that a token goes to: no other one's weights are read
        start, pair, place = _order(torch.searchsorted(used, s["topk"].long()), used.numel())

        def experts(m):
            codes, scales = (part.unflatten(0, (n, -1))[used] for part in m)
            return _values(codes, scales)

        x = s["x"].float()
        if c["act"] == "mx4":
            x = _values(*_quantise(x))
        g, u = _grouped(x[pair // K], start, experts(s["gate_up"])).split(c["I"], dim=1)
        h = g / (1 + torch.exp(-g)) * u
        if c["act"] == "mx4":
            h = _values(*_quantise(h))
        y = _grouped(h, start, experts(s["down"]))
        return (y[place].unflatten(0, (T, K)) * s["gates"][..., None]).sum(1).to(s["dt"])
    start, pair, place = _order(s["topk"], n)
    rows, gates = s["x"][pair // K], s["gates"]
    y = s["y"].float()[place].unflatten(0, (T, K))
    got = {"start": start.int(), "pair": pair.int(), "place": place.int(), "rows": rows,
           "out": (s["x"].float() + (y * gates[..., None]).sum(1)).to(s["dt"])}
    if c["grad"]:
        d = s["d_out"].float()
        got["d_y"] = (gates[..., None] * d[:, None]).flatten(0, 1)[pair].to(s["dt"])
        got["d_gates"] = (y * d[:, None]).sum(-1)
        got["d_x"] = s["d_in"].float()[place].unflatten(0, (T, K)).sum(1).to(s["dt"])
    return got


def run(s):
    if own:
        return _own(s)
    return _plain(s)


# ------------------------------------------------------- the framework's calls

def _plan(s):
    from paper_2607_24787_amd import spp
    c = s["case"]
    s["code"] = spp.DTYPE_BF16 if s["dt"] == torch.bfloat16 else spp.DTYPE_F32

    def matrix(codes, scales):
        return spp.make_mx4(codes.data_ptr(), scales.data_ptr(), codes.shape[0], 2 * codes.shape[1])

    size = 16
    if c["call"] == "quantize":
        s["matrix"] = matrix(s["codes"], s["scales"])
    elif c["call"] == "matmul":
        s["matrix"] = matrix(*s["w"])
        s["x_matrix"] = matrix(*s["xq"]) if c["act"] == "mx4" else None
    elif c["call"] == "experts":
        s["act"] = spp.ACT_MX4 if c["act"] == "mx4" else spp.ACT_BF16
        s["matrices"] = matrix(*s["gate_up"]), matrix(*s["down"])
        size = spp.spp_mx4_experts_workspace(c["n"], c["D"], c["I"], c["T"], c["K"])
    else:
        size = spp.spp_expert_sort_workspace(c["T"], c["K"], c["n"])
    s["workspace"] = torch.zeros(max(size, 16), dtype=torch.uint8, device=DEV)


def _own(s):
    from paper_2607_24787_amd import spp
    c = s["case"]
    stream = torch.cuda.current_stream().cuda_stream
    code, out, space = s["code"], s["out"], s["workspace"]
    if c["call"] == "quantize":
        spp.spp_mx4_quantize(code, s["x"].data_ptr(), c["cols"], s["matrix"], stream)
        spp.spp_mx4_load(s["matrix"], code, out.data_ptr(), c["cols"], stream)
        return out
    if c["call"] == "matmul":
        start = s["start"].data_ptr() if c["groups"] > 1 else 0
        if c["act"] == "mx4":
            spp.spp_mx4_matmul_mx4(s["matrix"], c["groups"], start, s["x_matrix"], c["M"], code, out.data_ptr(), c["N"],
                                   stream)
        else:
            spp.spp_mx4_matmul(s["matrix"], c["groups"], start, s["x"].data_ptr(), c["K"], c["M"], code, out.data_ptr(),
                               c["N"], stream)
        return out
    T, n, K, D = c["T"], c["n"], c["K"], c["D"]
    topk, gates, x = s["topk"].data_ptr(), s["gates"].data_ptr(), s["x"].data_ptr()
    if c["call"] == "experts":
        spp.spp_mx4_experts(*s["matrices"], n, s["act"], x, D, topk, gates, T, K, 0, 0, out.data_ptr(), D,
                            space.data_ptr(), space.numel(), stream)
        return out
    pair, place = s["pair"].data_ptr(), s["place"].data_ptr()
    spp.spp_expert_sort(topk, T, K, n, s["start"].data_ptr(), pair, place, space.data_ptr(), space.numel(), stream)
    spp.spp_expert_gather(code, x, D, place, T, K, D, s["rows"].data_ptr(), D, stream)
    spp.spp_expert_combine(code, s["y"].data_ptr(), D, place, gates, T, K, D, x, D, out.data_ptr(), D, stream)
    got = {k: s[k] for k in ("start", "pair", "place", "rows", "out")}
    if c["grad"]:
        spp.spp_expert_combine_grad(code, s["d_out"].data_ptr(), D, s["y"].data_ptr(), D, place, gates, T, K, D,
                                    s["d_y"].data_ptr(), D, s["d_gates"].data_ptr(), stream)
        spp.spp_expert_combine(code, s["d_in"].data_ptr(), D, place, 0, T, K, D, 0, 0, s["d_x"].data_ptr(), D, stream)
        got.update({k: s[k] for k in ("d_y", "d_gates", "d_x")})
    return got


# ----------------------------------------------------------------------- work

def _held(elements):
    return elements // 2 + elements // 32


def work(case):
    c = case
    elem = 2 if c["dtype"] == "bf16" else 4
    if c["call"] == "quantize":
        n = c["rows"] * c["cols"]
        return {"bytes": 2 * n * elem + 2 * _held(n), "flops": 3 * n}
    if c["call"] == "matmul":
        M, N, K, G = c["M"], c["N"], c["K"], c["groups"]
        x = _held(M * K) if c["act"] == "mx4" else 2 * M * K
        return {"bytes": min(G, M) * _held(N * K) + x + elem * M * N, "flops": 2 * M * N * K}
    T, n, K, D = c["T"], c["n"], c["K"], c["D"]
    P = T * K
    if c["call"] == "experts":
        distinct = n * (1 - (1 - K / n) ** T)
        return {"bytes": int(distinct * _held(3 * c["I"] * D)) + 4 * T * D + 8 * P, "flops": 6 * P * c["I"] * D}
    w = {"bytes": elem * (2 * T * D + 2 * P * D) + 16 * P + 4 * n, "flops": 2 * P * D}
    if c["grad"]:
        w = {"bytes": w["bytes"] + elem * (2 * T * D + 2 * P * D) + 4 * P, "flops": 6 * P * D}
    return w


# ---------------------------------------------------------------------- exact

def _decoded(matrix):
    """The values that codes and scales stand for, in 64 bits."""
    codes, scales = matrix
    i = torch.arange(2 * codes.shape[1], device=DEV)
    code = ((codes[:, i // 2] >> (4 * (i % 2)).to(torch.uint8)) & 15).double()
    size = code % 8
    size = torch.where(size < 2, size / 2, (1 + (size % 2) / 2) * torch.exp2(torch.floor(size / 2) - 1))
    return (1 - 2 * torch.floor(code / 8)) * size * torch.exp2(scales[:, i // 32].double() - 127)


def _nearest(y):
    """The values that 4 bits hold for y: per block of 32 the smallest power of two whose 7-fold is not below any
    magnitude, and the nearest of its multiples that a code names (ties to the even code)."""
    b = y.double().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True).clamp(min=7 * 2.0 ** -125)
    unit = torch.exp2(torch.ceil(torch.log2(top / 7)))
    a = b.abs() / unit
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (torch.sign(b) * (torch.round(a / step) * step).clamp(max=6.0) * unit).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]
    if c["call"] == "quantize":
        return torch.cat([_nearest(x) for x in s["x"].split(max(1, (1 << 25) // c["cols"]))])
    if c["call"] == "matmul":
        x = _decoded(s["xq"]) if c["act"] == "mx4" else s["x"].double()
        edge = s["start"].tolist()
        return torch.cat([x[edge[k]:edge[k + 1]] @ _decoded([m[k * c["N"]:(k + 1) * c["N"]] for m in s["w"]]).T
                          for k in range(c["groups"])])
    T, n, K, D = c["T"], c["n"], c["K"], c["D"]
    gates = s["gates"].double()
    if c["call"] == "experts":
        quantised = c["act"] == "mx4"
        x = _nearest(s["x"]) if quantised else s["x"].double()
        out = torch.zeros((T, D), dtype=torch.float64, device=DEV)
        for e in range(n):
            token, k = torch.nonzero(s["topk"] == e, as_tuple=True)
            gu = x[token] @ _decoded([m[e * 2 * c["I"]:(e + 1) * 2 * c["I"]] for m in s["gate_up"]]).T
            h = gu[:, :c["I"]] * torch.sigmoid(gu[:, :c["I"]]) * gu[:, c["I"]:]
            y = (_nearest(h) if quantised else h) @ _decoded([m[e * D:(e + 1) * D] for m in s["down"]]).T
            out.index_add_(0, token, y * gates[token, k][:, None])
        return out
    # where pair p = t K + k comes to stand: behind all pairs of lower experts, and those of its own before it
    flat = s["topk"].flatten().tolist()
    seen, first = [0] * n, [0] * (n + 1)
    for e in flat:
        first[e + 1] += 1
    for e in range(n):
        first[e + 1] += first[e]
    place = []
    for e in flat:
        place.append(first[e] + seen[e])
        seen[e] += 1
    place = torch.tensor(place, device=DEV).view(T, K)
    rows = torch.empty((T * K, D), dtype=torch.float64, device=DEV)
    rows[place] = s["x"].double()[:, None].expand(T, K, D)
    out, y = s["x"].double(), s["y"].double()
    for k in range(K):
        out = out + gates[:, k, None] * y[place[:, k]]
    got = {"start": None, "pair": None, "place": None, "rows": rows, "out": out}
    if c["grad"]:
        d, d_y = s["d_out"].double(), torch.empty_like(rows)
        d_gates, d_x = torch.empty_like(gates), torch.zeros_like(d)
        for k in range(K):
            d_y[place[:, k]] = gates[:, k, None] * d
            d_gates[:, k] = (d * y[place[:, k]]).sum(1)
            d_x = d_x + s["d_in"].double()[place[:, k]]
        got.update(d_y=d_y, d_gates=d_gates, d_x=d_x)
    return got
