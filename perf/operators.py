"""Operators of an expert layer in 8 bits, as cases that can be timed and compared.

Four operators, each a call or two of the public binding:

* ``dispatch``: tokens sorted by expert and their rows laid out in that order, in the tokens' type or in E4M3 with a scale
  per 128 values (``bsr_expert_sort`` with ``bsr_expert_scatter`` or ``bsr_expert_scatter_e4m3``); backward, the gradient of
  the tokens from that of the rows (``bsr_expert_combine`` without weights);
* ``combine``: the experts' outputs back per token, weighted and added to the residual stream (``bsr_expert_combine``);
  backward, the gradients of the rows and of the weights (``bsr_expert_combine_backward``);
* ``quantize``: rows in blocks of 1 x 128, or stacked weights in blocks of 128 x 128 with the transposed copies that
  gradients read (``bsr_quantize_e4m3_rows128``, ``bsr_quantize_e4m3_blocks128``);
* ``product``: the matrix product of such operands, dense or with a weight per expert's rows
  (``bsr_linear_forward_e4m3_block128``, ``bsr_expert_linear_e4m3_block128``).

A scale is a power of two, held as its exponent plus 127 in a byte; a row of scales is padded to a multiple of four bytes
(with 127) so that the scales of 512 values lie in one word.
"""
import math

import torch

own = False
binding = None


def listed():
    return [
        # one token of a batch of one in inference: latency
        dict(name="dispatch_1_token", op="dispatch", way="forward", tokens=1, top_k=4, experts=16, dim=384, dtype="bf16", e4m3=False, masked=0.0),
        # the expert layer of the small mixture model at its benchmark batch (64 images of 197 tokens), rows in 8 bits
        dict(name="dispatch_moe_vit_s_e4m3", op="dispatch", way="forward", tokens=12608, top_k=2, experts=16, dim=384, dtype="bf16", e4m3=True, masked=0.0),
        # a long batch through many small experts, a tenth of the tokens padding
        dict(name="dispatch_32768", op="dispatch", way="forward", tokens=32768, top_k=8, experts=128, dim=2048, dtype="bf16", e4m3=False, masked=0.1),
        # gradient of the tokens in the float32 configuration, odd sizes
        dict(name="dispatch_backward_fp32", op="dispatch", way="backward", tokens=6305, top_k=4, experts=23, dim=1028, dtype="fp32", e4m3=False, masked=0.02),
        # experts' outputs into the float residual stream of the small mixture model
        dict(name="combine_moe_vit_s", op="combine", way="forward", tokens=12608, top_k=2, experts=16, dim=384, dtype="bf16", out="fp32", masked=0.0),
        # gradient of the long batch's rows and weights
        dict(name="combine_backward_32768", op="combine", way="backward", tokens=32768, top_k=8, experts=128, dim=2048, dtype="bf16", out="bf16", masked=0.1),
        # activations of the base model at its benchmark batch (128 images of 197 tokens)
        dict(name="quantize_rows_vit_b", op="quantize", way="rows", m=25216, k=768, dtype="bf16"),
        # stacked weights of frozen experts with their transposed copies, sizes that are no multiples of 128
        dict(name="quantize_experts", op="quantize", way="blocks", experts=16, n=2000, k=1424, dtype="bf16", transposed=True),
        # QKV projection of the base model at its benchmark batch
        dict(name="linear_vit_b_qkv", op="product", way="linear", m=25216, n=2304, k=768, act=0, bias=True),
        # a large square-ish product
        dict(name="linear_8192", op="product", way="linear", m=8192, n=4096, k=7168, act=0, bias=False),
        # first layer of the small mixture model's experts: GELU, pre-activation kept for the backward pass
        dict(name="experts_moe_vit_s_gelu", op="product", way="experts", tokens=12608, top_k=2, experts=16, n=1536, k=384, act=1, bias=True, masked=0.0),
        # inference of a few tokens over many experts: every weight that is used is read once
        dict(name="experts_8_tokens", op="product", way="experts", tokens=8, top_k=8, experts=64, n=2048, k=1024, act=0, bias=True, masked=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["dispatch", "combine", "quantize", "product", "product"])
        masked = rng.choice([0.0, 0.0, 0.05, 0.3])
        if op in ("dispatch", "combine"):
            experts = _log(rng, 2, 256)
            dtype = rng.choice(["bf16", "bf16", "fp32"])
            case = dict(op=op, way=rng.choice(["forward", "backward"]), tokens=_log(rng, 1, 32768), top_k=min(experts, rng.randint(1, 8)), experts=experts,
                        dim=8 * _log(rng, 4, 512), dtype=dtype, masked=masked)
            if op == "dispatch":
                case["e4m3"] = case["way"] == "forward" and rng.random() < 0.5
                if case["e4m3"]:
                    case["dim"] = max(16, case["dim"] // 16 * 16)
            else:
                case["out"] = rng.choice(["bf16", "fp32"])
        elif op == "quantize" and rng.random() < 0.5:
            case = dict(op=op, way="rows", m=_log(rng, 1, 65536), k=16 * _log(rng, 1, 512), dtype=rng.choice(["bf16", "bf16", "fp32"]))
        elif op == "quantize":
            case = dict(op=op, way="blocks", experts=_log(rng, 1, 64), n=16 * _log(rng, 1, 256), k=16 * _log(rng, 1, 256), dtype=rng.choice(["bf16", "bf16", "fp32"]),
                        transposed=rng.random() < 0.7)
        else:
            act = rng.choice([0, 0, 1, 2])
            case = dict(op=op, way=rng.choice(["linear", "experts"]), n=8 * _log(rng, 8, 512), k=16 * _log(rng, 4, 448), act=act, bias=act != 2 and rng.random() < 0.5)
            if case["way"] == "linear":
                case["m"] = _log(rng, 1, 32768)
            else:
                case["experts"] = _log(rng, 2, 128)
                case["top_k"] = min(case["experts"], rng.randint(1, 8))
                case["tokens"] = _log(rng, 1, 8192)
                case["masked"] = masked
        if _cost(case) <= most and _held(case) < 6e9:
            return case


def _cost(case):
    """Seconds at round figures for the card's bf16 and memory rates."""
    w = work(case)
    return max(w["flops"] / 1.6e15, w["bytes"] / 6.5e12)


def _held(case):
    """Bytes of the largest intermediate that the plain form holds in 32 bits."""
    if case["op"] in ("dispatch", "combine"):
        return 4 * case["tokens"] * case["top_k"] * case["dim"]
    if case["op"] == "quantize":
        return 4 * case["k"] * (case["m"] if case["way"] == "rows" else case["n"] * case["experts"])
    return 4 * (case.get("experts", 1) * case["n"] * case["k"] + _rows(case) * (case["n"] + case["k"]))


SIZE = {"bf16": 2, "fp32": 4}
TYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _rows(case):
    return case["m"] if "m" in case else case["tokens"] * case["top_k"]


def work(case):
    op, way = case["op"], case["way"]
    if op in ("dispatch", "combine"):
        t, slots, d, b = case["tokens"], case["tokens"] * case["top_k"], case["dim"], SIZE[case["dtype"]]
        rows = int(slots * (1.0 - case["masked"]))
        if op == "dispatch" and way == "forward":
            out = rows * (d + _scales(d)) if case["e4m3"] else rows * d * b
            return dict(bytes=8 * slots + 4 * (case["experts"] + 1) + t * d * b + out, flops=t * d if case["e4m3"] else 0)
        if op == "dispatch":
            return dict(bytes=4 * slots + rows * d * b + t * d * b, flops=rows * d)
        o = SIZE[case["out"]]
        if way == "forward":
            return dict(bytes=8 * slots + rows * d * b + 2 * t * d * o, flops=2 * rows * d)
        return dict(bytes=12 * slots + 2 * rows * d * b + t * d * o, flops=3 * rows * d)
    if op == "quantize":
        k, b = case["k"], SIZE[case["dtype"]]
        if way == "rows":
            return dict(bytes=case["m"] * (k * b + k + _scales(k)), flops=2 * case["m"] * k)
        n, e = case["n"], case["experts"]
        out = n * k + -(-n // 128) * _scales(k)
        if case["transposed"]:
            out += n * k + -(-k // 128) * _scales(n)
        return dict(bytes=e * (n * k * b + out), flops=2 * e * n * k)
    n, k = case["n"], case["k"]
    rows = case["m"] if way == "linear" else int(_rows(case) * (1.0 - case["masked"]))
    weights = 1 if way == "linear" else min(case["experts"], rows)
    y = rows * n * (4 if case["act"] else 2)        # with the pre-activation
    return dict(bytes=rows * (k + _scales(k)) + weights * (n * k + -(-n // 128) * _scales(k) + (4 * n if case["bias"] else 0)) + y, flops=2 * rows * n * k)


def _scales(k):
    """Bytes of a row of scales over k values."""
    return 4 * -(-k // 512)


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _values(gen, shape, dtype, spread=1.0):
    """Activations: normal, with a size of its own for every row and a few channels that are much larger than the others."""
    x = torch.randn(shape, generator=gen, device="cuda")
    x = x * torch.exp(0.5 * torch.randn(shape[:-1] + (1,), generator=gen, device="cuda"))
    loud = torch.rand(shape[-1], generator=gen, device="cuda") < 0.01
    return (x * torch.where(loud, 12.0, 1.0) * spread).to(dtype)


def _routing(gen, tokens, top_k, experts, masked):
    """What a router gives: distinct experts for every token, some more popular than others, the weights a softmax over the chosen
    logits; slots of padded tokens have expert -1."""
    logits = torch.randn((tokens, experts), generator=gen, device="cuda") + 0.7 * torch.randn((1, experts), generator=gen, device="cuda")
    top, expert = torch.topk(logits, top_k, dim=1)
    pad = torch.rand((tokens, 1), generator=gen, device="cuda") < masked
    return torch.where(pad, -1, expert).to(torch.int32).contiguous(), torch.softmax(top, dim=1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op, way = case["op"], case["way"]
    s = dict(case=case)
    if op in ("dispatch", "combine"):
        t, top_k, d, dtype = case["tokens"], case["top_k"], case["dim"], TYPE[case["dtype"]]
        s["expert"], s["weights"] = _routing(gen, t, top_k, case["experts"], case["masked"])
        slots = t * top_k
        if op == "dispatch" and way == "forward":
            s["x"] = _values(gen, (t, d), dtype)
            s["pos"] = torch.empty((t, top_k), dtype=torch.int32, device="cuda")
            s["seg"] = torch.empty(case["experts"] + 1, dtype=torch.int32, device="cuda")
            if case["e4m3"]:
                s["q"] = torch.zeros((slots, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
                s["scale"] = torch.zeros((slots, _scales(d)), dtype=torch.uint8, device="cuda")
            else:
                s["rows"] = torch.zeros((slots, d), dtype=dtype, device="cuda")
            return s
        s["pos"], s["seg"] = _sort(s["expert"], case["experts"])
        s["rows"] = _values(gen, (slots, d), dtype)
        if op == "dispatch":
            s["dx"] = torch.empty((t, d), dtype=dtype, device="cuda")
        elif way == "forward":
            s["residual"] = _values(gen, (t, d), TYPE[case["out"]])
            s["out"] = torch.empty((t, d), dtype=TYPE[case["out"]], device="cuda")
        else:
            s["dout"] = _values(gen, (t, d), TYPE[case["out"]], 1e-2)
            s["drows"] = torch.zeros((slots, d), dtype=dtype, device="cuda")
            s["dw"] = torch.empty((t, top_k), dtype=torch.float32, device="cuda")
        return s
    if op == "quantize":
        k, dtype = case["k"], TYPE[case["dtype"]]
        if way == "rows":
            m = case["m"]
            s["x"] = _values(gen, (m, k), dtype)
            s["q"] = torch.empty((m, k), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            s["scale"] = torch.empty((m, _scales(k)), dtype=torch.uint8, device="cuda")
            return s
        e, n = case["experts"], case["n"]
        s["w"] = _values(gen, (e, n, k), dtype, 0.02)
        s["q"] = torch.empty((e, n, k), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        s["scale"] = torch.empty((e, -(-n // 128), _scales(k)), dtype=torch.uint8, device="cuda")
        s["qt"] = s["scale_t"] = None
        if case["transposed"]:
            s["qt"] = torch.empty((e, k, n), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            s["scale_t"] = torch.empty((e, -(-k // 128), _scales(n)), dtype=torch.uint8, device="cuda")
        return s
    n, k, rows = case["n"], case["k"], _rows(case)
    stack = (n, k) if way == "linear" else (case["experts"], n, k)
    s["xq"], s["xs"] = _quantize_rows(_values(gen, (rows, k), torch.bfloat16))
    s["wq"], s["ws"] = _quantize_blocks((torch.randn(stack, generator=gen, device="cuda") / math.sqrt(k)).to(torch.bfloat16))
    s["bias"] = 0.1 * torch.randn(stack[:-1], generator=gen, device="cuda") if case["bias"] else None
    s["y"] = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
    s["z"] = None
    if case["act"] == 1:
        s["z"] = torch.zeros((rows, n), dtype=torch.bfloat16, device="cuda")
    elif case["act"] == 2:
        s["z"] = _values(gen, (rows, n), torch.bfloat16)
    if way == "experts":
        expert, _ = _routing(gen, case["tokens"], case["top_k"], case["experts"], case["masked"])
        _, s["seg"] = _sort(expert, case["experts"])
        s["ends"] = s["seg"].tolist()            # a program of plain calls has to know the segments on the host
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(s):
    global binding
    if own and binding is None:
        from paper_2405_10951_b200 import binding
    return RUN[s["case"]["op"], s["case"]["way"]](s)


def _run_dispatch(s):
    if own:
        binding.bsr_expert_sort(s["expert"], s["case"]["experts"], pos=s["pos"], seg_start=s["seg"])
        if s["case"]["e4m3"]:
            binding.bsr_expert_scatter_e4m3(s["x"], s["pos"], q=s["q"], scale=s["scale"])
            return [s["pos"], s["seg"], s["q"], s["scale"]]
        binding.bsr_expert_scatter(s["x"], s["pos"], rows=s["rows"])
        return [s["pos"], s["seg"], s["rows"]]
    pos, seg = _sort(s["expert"], s["case"]["experts"])
    used = (pos >= 0).reshape(-1)
    to = pos.reshape(-1)[used].long()
    token = torch.div(torch.arange(used.numel(), device="cuda"), s["case"]["top_k"], rounding_mode="floor")[used]
    if s["case"]["e4m3"]:
        q, scale = _quantize_rows(s["x"])
        s["q"].view(torch.uint8)[to] = q.view(torch.uint8)[token]
        s["scale"][to] = scale[token]
        return [pos, seg, s["q"], s["scale"]]
    s["rows"][to] = s["x"][token]
    return [pos, seg, s["rows"]]


def _run_dispatch_backward(s):
    if own:
        return binding.bsr_expert_combine(s["rows"], s["pos"], out=s["dx"])
    return _weighted(s["rows"], s["pos"], None).to(s["dx"].dtype)


def _run_combine(s):
    if own:
        return binding.bsr_expert_combine(s["rows"], s["pos"], s["weights"], residual=s["residual"], out=s["out"])
    return (s["residual"].float() + _weighted(s["rows"], s["pos"], s["weights"])).to(s["out"].dtype)


def _run_combine_backward(s):
    if own:
        return binding.bsr_expert_combine_backward(s["dout"], s["rows"], s["pos"], s["weights"], drows=s["drows"], dw=s["dw"])
    dout, used = s["dout"].float(), s["pos"] >= 0
    rows = s["rows"][s["pos"].clamp(min=0).long()].float()
    dw = torch.where(used, (rows * dout[:, None, :]).sum(-1), 0.0)
    g = (s["weights"][..., None] * dout[:, None, :]).to(s["drows"].dtype)
    s["drows"][s["pos"][used].long()] = g[used]
    return s["drows"], dw


def _run_quantize_rows(s):
    if own:
        return binding.bsr_quantize_e4m3_rows128(s["x"], q=s["q"], scale=s["scale"])
    return _quantize_rows(s["x"])


def _run_quantize_blocks(s):
    if own:
        return binding.bsr_quantize_e4m3_blocks128(s["w"], q=s["q"], scale=s["scale"], qt=s["qt"], scale_t=s["scale_t"])
    out = _quantize_blocks(s["w"])
    return out + _quantize_blocks(s["w"].transpose(1, 2)) if s["case"]["transposed"] else out


def _run_linear(s):
    if own:
        y = binding.bsr_linear_forward_e4m3_block128(s["xq"], s["xs"], s["wq"], s["ws"], s["bias"], act=s["case"]["act"], z=s["z"], y=s["y"])
        return [y, s["z"]] if s["case"]["act"] == 1 else y
    acc = _rows_float(s["xq"], s["xs"]) @ _blocks_float(s["wq"], s["ws"]).t()
    return _epilogue(s, acc)


def _run_experts(s):
    if own:
        y = binding.bsr_expert_linear_e4m3_block128(s["xq"], s["xs"], s["wq"], s["ws"], s["seg"], s["bias"], act=s["case"]["act"], z=s["z"], y=s["y"])
        return [y, s["z"]] if s["case"]["act"] == 1 else y
    x, w = _rows_float(s["xq"], s["xs"]), _blocks_float(s["wq"], s["ws"])
    acc = torch.zeros(s["y"].shape, dtype=torch.float32, device="cuda")
    for e in range(s["case"]["experts"]):
        a, b = s["ends"][e], s["ends"][e + 1]
        if a < b:
            torch.matmul(x[a:b], w[e].t(), out=acc[a:b])
    return _epilogue(s, acc, torch.searchsorted(s["seg"][1:].contiguous(), torch.arange(x.shape[0], device="cuda", dtype=torch.int32), right=True))


RUN = {("dispatch", "forward"): _run_dispatch, ("dispatch", "backward"): _run_dispatch_backward, ("combine", "forward"): _run_combine,
       ("combine", "backward"): _run_combine_backward, ("quantize", "rows"): _run_quantize_rows, ("quantize", "blocks"): _run_quantize_blocks,
       ("product", "linear"): _run_linear, ("product", "experts"): _run_experts}


# ---- plain forms -------------------------------------------------------------------------------------------------------
def _sort(expert, experts):
    flat = expert.reshape(-1).long()
    used = (flat >= 0) & (flat < experts)
    key = torch.where(used, flat, experts)
    order = torch.argsort(key, stable=True)
    pos = torch.empty_like(order)
    pos[order] = torch.arange(order.numel(), device=order.device)
    pos = torch.where(used, pos, -1)
    seg = torch.zeros(experts + 1, dtype=torch.int32, device=expert.device)
    seg[1:] = torch.cumsum(torch.bincount(key, minlength=experts + 1)[:experts], 0)
    return pos.reshape(expert.shape).to(torch.int32), seg


def _weighted(rows, pos, weights):
    got = rows[pos.clamp(min=0).long()].float()
    if weights is not None:
        got = got * weights[..., None]
    return torch.where((pos >= 0)[..., None], got, 0.0).sum(1)


def _exponent(amax):
    """The least e with amax <= 448 * 2^e (448 = 0.875 * 2^9), at least -127; 0 for a block of zeros."""
    f, p = torch.frexp(amax)
    e = torch.clamp(p - 9 + (f > 0.875).to(p.dtype), min=-127)
    return torch.where(amax > 0, e, 0)


def _power(e):
    """2^e, exact, for -127 <= e <= 127."""
    return ((torch.clamp(e, min=-126).to(torch.int32) + 127) << 23).view(torch.float32) * torch.where(e < -126, 0.5, 1.0)


def _quantize_rows(x):
    m, k = x.shape
    kb = -(-k // 128)
    v = torch.nn.functional.pad(x.float(), (0, kb * 128 - k)).view(m, kb, 128)
    e = _exponent(v.abs().amax(-1))
    q = (v * _power(-e[..., None])).view(m, kb * 128)[:, :k].contiguous().to(torch.float8_e4m3fn)
    scale = torch.nn.functional.pad(e + 127, (0, _scales(k) - kb), value=127)
    return q, scale.to(torch.uint8)


def _quantize_blocks(w):
    n, k = w.shape[-2:]
    stack = w.reshape(-1, n, k)
    nb, kb = -(-n // 128), -(-k // 128)
    v = torch.nn.functional.pad(stack.float(), (0, kb * 128 - k, 0, nb * 128 - n)).view(-1, nb, 128, kb, 128)
    e = _exponent(v.abs().amax((2, 4)))
    q = (v * _power(-e[:, :, None, :, None])).view(-1, nb * 128, kb * 128)[:, :n, :k].contiguous().to(torch.float8_e4m3fn)
    scale = torch.nn.functional.pad(e + 127, (0, _scales(k) - kb), value=127)
    return q.view(w.shape), scale.to(torch.uint8).view(w.shape[:-2] + (nb, _scales(k)))


def _rows_float(q, scale):
    k = q.shape[1]
    e = scale.int().repeat_interleave(128, 1)[:, :k] - 127
    return q.float() * _power(e)


def _blocks_float(q, scale):
    n, k = q.shape[-2:]
    e = scale.int().repeat_interleave(128, -2)[..., :n, :].repeat_interleave(128, -1)[..., :k] - 127
    return q.float() * _power(e)


def _epilogue(s, acc, expert=None):
    """Bias and activation in 32 bits; rows behind the last segment stay as they were."""
    case = s["case"]
    if s["bias"] is not None:
        acc = acc + (s["bias"] if expert is None else s["bias"][expert.clamp(max=case["experts"] - 1)])
    z = None
    if case["act"] == 1:
        z = acc.to(torch.bfloat16)
        acc = acc * 0.5 * (1.0 + torch.erf(acc * math.sqrt(0.5)))
    elif case["act"] == 2:
        v = s["z"].float()
        acc = acc * (0.5 * (1.0 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi))
    y = acc.to(s["y"].dtype)
    if expert is not None:
        used = (expert < case["experts"])[:, None]
        y = torch.where(used, y, s["y"])
        z = torch.where(used, z, s["z"]) if z is not None else None
    return y if z is None else [y, z]


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    op, way = case["op"], case["way"]
    if op == "dispatch" and way == "forward":
        if case["e4m3"]:
            block = torch.nn.functional.pad(s["x"].double(), (0, -case["dim"] % 128)).unflatten(1, (-1, 128))
            code = _codes(block, block.abs().amax(-1, keepdim=True)).flatten(1)[:, :case["dim"]]
            return [None, None, _placed(s, code), None]
        return [None, None, _placed(s, s["x"].double())]
    if op == "dispatch":
        return _sum_of_slots(s, torch.ones_like(s["weights"], dtype=torch.float64))
    if op == "combine" and way == "forward":
        return s["residual"].double() + _sum_of_slots(s, s["weights"].double())
    if op == "combine":
        slot = _slots(s)
        g = s["dout"].double()[slot // case["top_k"]]
        drows, dw = s["drows"].double(), torch.zeros(s["weights"].numel(), dtype=torch.float64, device="cuda")
        drows[:len(slot)] = s["weights"].double().reshape(-1, 1)[slot] * g
        dw[slot] = torch.einsum("rd,rd->r", g, s["rows"][:len(slot)].double())
        return drows, dw.view(s["weights"].shape)
    if op == "quantize" and way == "rows":
        block = torch.nn.functional.pad(s["x"].double(), (0, -case["k"] % 128)).unflatten(1, (-1, 128))
        return _codes(block, block.abs().amax(-1, keepdim=True)).flatten(1)[:, :case["k"]], None
    if op == "quantize":
        q = _weight_codes(s["w"].double())
        return (q, None, _weight_codes(s["w"].double().transpose(1, 2)), None) if case["transposed"] else (q, None)
    x = torch.nn.functional.pad(s["xq"].double(), (0, -case["k"] % 128)).unflatten(1, (-1, 128))
    x = (x * _two(s["xs"][:, :x.shape[1], None].int() - 127)).flatten(1)[:, :case["k"]]
    w = torch.nn.functional.pad(s["wq"].double(), (0, -case["k"] % 128, 0, -case["n"] % 128)).unflatten(-1, (-1, 128)).unflatten(-3, (-1, 128))
    w = (w * _two(s["ws"][..., :w.shape[-2]].int() - 127)[..., None, :, None]).flatten(-2).flatten(-3, -2)[..., :case["n"], :case["k"]]
    y = s["y"].double()
    z = s["z"].double() if case["act"] == 1 else None
    parts = [(0, case["m"], w, s["bias"])] if way == "linear" else [
        (s["ends"][e], s["ends"][e + 1], w[e], None if s["bias"] is None else s["bias"][e]) for e in range(case["experts"])]
    for a, b, we, be in parts:
        part = x[a:b] @ we.t()
        if be is not None:
            part = part + be.double()
        normal = torch.distributions.Normal(torch.zeros((), dtype=torch.float64, device="cuda"), 1.0)
        if case["act"] == 1:
            z[a:b] = part
            part = part * normal.cdf(part)
        elif case["act"] == 2:
            v = s["z"][a:b].double()
            part = part * (normal.cdf(v) + v * torch.exp(normal.log_prob(v)))
        y[a:b] = part
    return y if z is None else [y, z]


def _slots(s):
    """The slots that have an expert, in the order of their rows."""
    flat = s["expert"].reshape(-1).long()
    slot = torch.nonzero((flat >= 0) & (flat < s["case"]["experts"])).squeeze(1)
    return slot[torch.sort(flat[slot] * flat.numel() + slot).indices]


def _placed(s, x):
    slot = _slots(s)
    rows = torch.zeros((s["expert"].numel(), x.shape[1]), dtype=torch.float64, device="cuda")
    rows[:len(slot)] = x[slot // s["case"]["top_k"]]
    return rows


def _sum_of_slots(s, weights):
    slot = _slots(s)
    out = torch.zeros((s["case"]["tokens"], s["case"]["dim"]), dtype=torch.float64, device="cuda")
    return out.index_add(0, slot // s["case"]["top_k"], weights.reshape(-1, 1)[slot] * s["rows"][:len(slot)].double())


def _two(e):
    """2^e in 64 bits, from the bits of its exponent (the device's pow may be off in its last place)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _codes(v, amax):
    """E4M3 values of v over its block's scale: three bits behind the leading one, steps of 2^-9 below 2^-6, to nearest and even."""
    tight = torch.where(amax > 0, amax, 448.0) / 448.0
    e = torch.clamp(torch.ceil(torch.log2(tight)), min=-127.0)
    e = torch.where(_two(e) < tight, e + 1, torch.where((_two(e - 1) >= tight) & (e > -127), e - 1, e))
    u = v / _two(e)
    step = _two(torch.clamp(torch.frexp(u).exponent - 1, min=-6, max=8) - 3)
    return torch.round(u / step) * step


def _weight_codes(w):
    n, k = w.shape[-2:]
    v = torch.nn.functional.pad(w, (0, -k % 128, 0, -n % 128)).unflatten(2, (-1, 128)).unflatten(1, (-1, 128))
    return _codes(v, v.abs().amax((2, 4), keepdim=True)).flatten(3, 4).flatten(1, 2)[:, :n, :k]
