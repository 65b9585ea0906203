"""The ends of a training step around the head, as sized calls: byte embeddings, the residual norm, the gradients' norm.

The head reads hidden states and returns gradients. What a model trained with it does just before and just after:
  embed      rows of the byte embedding, scaled: out[t] = scale * table[token[t]]; a negative token (padding) is a row of zeros
  embed_grad its gradient: d_table[b] = scale * sum of d_out[t] over the positions with token b; every row is written
  norm       s = x + residual; out = s / sqrt(mean(s^2) + eps) * weight; s itself, the residual stream, is returned too. With
             `bits8` the output is held in e4m3 with a scale per row or per `group` columns: amax / 448, and out / scale in 8 bits
  norm_grad  from the gradient of out (the head's d_hidden, fp32) and of s (the residual stream's, optional): the gradient of s,
             which is that of x and of residual, and of the weight
  clip       the 2-norm of all gradients of a model together, and the gradients scaled to `max_norm` where it is larger
Inputs are synthetic: Zipf-distributed tokens with padding behind every text, activations ~N(0,1) with a few large columns as
trained models have, weights near one, gradients ~N(0, std).
"""
from __future__ import annotations

import math

import torch

own = False
EPS = 1e-5

# Sizes of the parameter gradients of a head: (n, r, v, d) of its unembeddings, the rank of its adaptors (0: composed).
_HEADS = {"dense": (8, 16, 320, 4096, 0), "factored": (8, 16, 320, 4096, 16), "small": (4, 8, 256, 256, 0)}


def listed():
    return [
        # one step of 64 sequences being decoded: the bytes that were accepted last, as the next inputs
        dict(op="embed", name="embed_step_64", seqs=64, length=1, v=320, d=4096, table="bf16", out="bf16"),
        # a training batch of 16 texts of 4096 bytes
        dict(op="embed", name="embed_text_65536", seqs=16, length=4096, v=320, d=4096, table="bf16", out="bf16"),
        # the embedding's gradient in the training step of the benchmark's head: few symbols, many positions each
        dict(op="embed_grad", name="embed_grad_8192", seqs=8, length=1024, v=320, d=4096, grad="f32"),
        # an uneven batch on a large vocabulary: most rows of the gradient are zeros
        dict(op="embed_grad", name="embed_grad_wide_2005", seqs=5, length=401, v=32768, d=2048, grad="bf16"),
        # one sequence being decoded: the residual stream's last addition and the norm in front of the head
        dict(op="norm", name="norm_step_1", rows=1, d=4096, io="bf16", pad=0, bits8=False, group=0),
        # the same for a training batch
        dict(op="norm", name="norm_8192", rows=8192, d=4096, io="bf16", pad=0, bits8=False, group=0),
        # hidden states for an 8-bit product, scales per 128 columns, from rows of a wider buffer
        dict(op="norm", name="norm_bits8_2005", rows=2005, d=4096, io="bf16", pad=64, bits8=True, group=128),
        # the norm's gradient behind the head's training call
        dict(op="norm_grad", name="norm_grad_8192", rows=8192, d=4096, io="bf16", dx="bf16", stream=True),
        # fp32 activations of an odd width
        dict(op="norm_grad", name="norm_grad_odd_693", rows=693, d=1001, io="f32", dx="f32", stream=False),
        # all gradients of the benchmark's head with its unembeddings composed
        dict(op="clip", name="clip_dense", head="dense", many=0, dtype="f32", std=1e-3, max_norm=1.0),
        # the same head with shared unembeddings and adaptors
        dict(op="clip", name="clip_factored", head="factored", many=0, dtype="f32", std=1e-3, max_norm=1.0),
        # a small head beside the many small tensors (norms, biases, adaptors) of a model, packed one behind the other
        dict(op="clip", name="clip_many", head="small", many=600, dtype="bf16", std=1e-3, max_norm=0.5),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["embed", "embed_grad", "norm", "norm_grad", "clip"])
    d = _log_uniform(rng, 64, 8192)
    if rng.random() < 0.75:
        d = (d + 7) // 8 * 8
    dtype = rng.choice(["bf16", "f32"])
    if op in ("embed", "embed_grad"):
        v = rng.choice([256, 268, 320, _log_uniform(rng, 2, 32768)])
        v = min(v, (32768 * 2048) // d)
        most = (65536 * 4096 if op == "embed" else 8192 * 4096) // d
        rows = _log_uniform(rng, 1, min(65536, most))
        seqs = rng.randint(1, min(16, rows))
        case = dict(op=op, seqs=seqs, length=max(1, rows // seqs), v=v, d=d)
        return dict(case, table=dtype, out=rng.choice(["bf16", dtype])) if op == "embed" else dict(case, grad=dtype)
    if op == "clip":
        return dict(op=op, head=rng.choice(["factored", "small", "small"]), many=rng.choice([0, _log_uniform(rng, 1, 1000)]), dtype=dtype,
                    std=math.exp(rng.uniform(math.log(1e-6), math.log(1e-1))), max_norm=rng.choice([0.1, 0.5, 1.0, 10.0]))
    rows = _log_uniform(rng, 1, min(16384, 8192 * 4096 // d))
    if op == "norm":
        return dict(op=op, rows=rows, d=d, io=dtype, pad=rng.choice([0, 0, 8, 64]), bits8=rng.random() < 0.4, group=rng.choice([0, 32, 128]))
    return dict(op=op, rows=rows, d=d, io=dtype, dx=rng.choice(["bf16", dtype]), stream=rng.random() < 0.5)


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _tokens(case, g):
    """Zipf-distributed symbols of `seqs` texts, the last twentieth of each padding (-1)."""
    seqs, length, v = case["seqs"], case["length"], case["v"]
    weight = 1.0 / torch.arange(1, v + 1, device="cuda", dtype=torch.float32) ** 1.1
    order = torch.randperm(v, device="cuda", generator=g)
    text = order[torch.multinomial(weight, seqs * length, replacement=True, generator=g)].view(seqs, length)
    text[:, length - length // 20:] = -1
    return text.reshape(-1).to(torch.int32)


def _sizes(case):
    """Elements of every gradient tensor: (fp32 ones of the head, the model's small ones of the case's type)."""
    n, r, v, d, k = _HEADS[case["head"]]
    head = [n * v * d, n * r * v * k, n * r * k * d, r * d] if k else [n * r * v * d, r * d]
    return head, [1 + (i * 7919) % 4099 for i in range(case["many"])]


class _State:
    pass


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    s = _State()
    s.case, s.plan = case, None
    op = case["op"]
    if op in ("embed", "embed_grad"):
        s.tokens = _tokens(case, g)
        T, v, d = s.tokens.numel(), case["v"], case["d"]
        s.scale = math.sqrt(d)
        if op == "embed":
            s.table = normal(v, d, std=0.02, dtype=_dtype(case["table"]))
            s.out = empty(T, d, dtype=_dtype(case["out"]))
        else:
            s.d_out = normal(T, d, std=1e-3, dtype=_dtype(case["grad"]))
            s.d_table = empty(v, d)
    elif op in ("norm", "norm_grad"):
        T, d, io = case["rows"], case["d"], _dtype(case["io"])
        large = 1.0 + 15.0 * (torch.rand(d, device="cuda", generator=g) < 0.01)       # a few columns of large values
        pad = case.get("pad", 0)
        s.x = torch.cat([normal(T, d) * large, normal(T, pad)], 1).to(io)[:, :d]      # rows `pad` elements further apart than wide
        s.weight = (1.0 + 0.1 * normal(d)).to(io)
        if op == "norm":
            s.residual = normal(T, d, dtype=io)
            s.out_sum = empty(T, d, dtype=io)
            if case["bits8"]:
                groups = -(-d // case["group"]) if case["group"] else 1
                s.out_q, s.out_scale = empty(T, d, dtype=torch.float8_e4m3fn), empty(T, groups)
            else:
                s.out = empty(T, d, dtype=io)
        else:
            s.d_out = normal(T, d, std=1e-3)
            s.d_sum = normal(T, d, std=1e-3, dtype=_dtype(case["dx"])) if case["stream"] else None
            s.d_x, s.d_weight = empty(T, d, dtype=_dtype(case["dx"])), empty(d)
    else:
        head, small = _sizes(case)
        # the head's gradients start on multiples of 512 bytes as an allocator gives them, zeros between them; the small ones are packed
        at, places = 0, []
        for c in head:
            places.append((at, c))
            at = (at + c + 127) // 128 * 128
        s.head = torch.zeros(at, device="cuda")
        for o, c in places:
            s.head[o:o + c].normal_(0.0, case["std"], generator=g)
        s.small = normal(sum(small), std=case["std"], dtype=_dtype(case["dtype"]))
        s.head_out, s.small_out = torch.zeros_like(s.head), torch.empty_like(s.small)
        s.grads = [s.head[o:o + c] for o, c in places] + list(torch.split(s.small, small) if small else [])
        s.outs = [s.head_out[o:o + c] for o, c in places] + list(torch.split(s.small_out, small) if small else [])
        s.norm = empty(1)
    return s


def run(s):
    case, op = s.case, s.case["op"]
    if own:
        from paper_2511_11346_b200 import binding
        if op == "embed":
            binding.mtpc_embed(s.tokens, s.table, s.out, scale=s.scale)
            return [s.out]
        if op == "embed_grad":
            binding.mtpc_embed_backward(s.tokens, s.d_out, s.d_table, scale=s.scale)
            return [s.d_table]
        if op == "norm" and case["bits8"]:
            binding.mtpc_residual_rmsnorm(s.x, s.residual, s.weight, EPS, None, out_sum=s.out_sum, out_q=s.out_q, out_scale=s.out_scale,
                                          scale_group=case["group"])
            return [s.out_sum, s.out_q, s.out_scale]
        if op == "norm":
            binding.mtpc_residual_rmsnorm(s.x, s.residual, s.weight, EPS, s.out, out_sum=s.out_sum)
            return [s.out_sum, s.out]
        if op == "norm_grad":
            binding.mtpc_residual_rmsnorm_backward(s.x, s.weight, EPS, s.d_out, s.d_sum, s.d_x, s.d_weight)
            return [s.d_x, s.d_weight]
        if s.plan is None:                        # a training loop's gradients stay where they are: it makes the list once
            s.plan = binding.GradientList(s.grads, s.outs)
        s.plan.mtpc_clip_gradients(case["max_norm"], s.norm)
        return [s.norm, s.head_out, s.small_out]

    if op == "embed":
        rows = s.table[s.tokens.clamp_min(0).long()].float() * s.scale
        return [torch.where(s.tokens[:, None] < 0, 0.0, rows).to(s.out.dtype)]
    if op == "embed_grad":
        keep = s.tokens >= 0
        d_table = torch.zeros_like(s.d_table)
        d_table.index_add_(0, s.tokens[keep].long(), s.d_out[keep].float())
        return [d_table * s.scale]
    if op == "norm":
        x = s.x.float() + s.residual.float()
        y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * s.weight.float()
        if not case["bits8"]:
            return [x.to(s.x.dtype), y.to(s.x.dtype)]
        scale = _by_group(y.abs(), case).amax(2) / 448.0
        scale = torch.where(scale == 0, 1.0, scale)
        codes = (_by_group(y, case) / scale[:, :, None]).clamp(-448.0, 448.0).flatten(1)[:, :case["d"]].to(torch.float8_e4m3fn)
        return [x.to(s.x.dtype), codes, scale]
    if op == "norm_grad":
        x, w, dy = s.x.float(), s.weight.float(), s.d_out
        rstd = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
        dx = rstd * (dy * w - x * rstd * rstd * (dy * w * x).mean(1, keepdim=True))
        if s.d_sum is not None:
            dx = dx + s.d_sum.float()
        return [dx.to(s.d_x.dtype), (dy * x * rstd).sum(0)]
    norm = torch.sqrt(s.head.square().sum(dtype=torch.float64) + s.small.float().square().sum(dtype=torch.float64))
    c = torch.where(norm > case["max_norm"], case["max_norm"] / norm, 1.0).float()
    return [norm.float().reshape(1), s.head * c, (s.small.float() * c).to(s.small.dtype)]


def _by_group(y, case):
    """[T, d] -> [T, groups, columns of a group], zeros behind a last short one."""
    group = case["group"] or case["d"]
    return torch.nn.functional.pad(y, (0, -case["d"] % group)).unflatten(1, (-1, group))


def work(case):
    op, size = case["op"], {"f32": 4, "bf16": 2}
    if op == "embed":                             # the tokens, the table's rows that are asked for, the output
        T, v, d = case["seqs"] * case["length"], case["v"], case["d"]
        return {"bytes": 4 * T + min(T, v) * d * size[case["table"]] + T * d * size[case["out"]], "flops": T * d}
    if op == "embed_grad":
        T, v, d = case["seqs"] * case["length"], case["v"], case["d"]
        return {"bytes": 4 * T + T * d * size[case["grad"]] + 4 * v * d, "flops": T * d}
    if op == "norm":
        T, d, b = case["rows"], case["d"], size[case["io"]]
        groups = -(-d // case["group"]) if case["group"] else 1
        out = T * d + 4 * T * groups if case["bits8"] else T * d * b
        return {"bytes": 3 * T * d * b + d * b + out, "flops": 5 * T * d}
    if op == "norm_grad":
        T, d, b = case["rows"], case["d"], size[case["io"]]
        return {"bytes": T * d * (b + 4 + size[case["dx"]] * (2 if case["stream"] else 1)) + d * (b + 4), "flops": 10 * T * d}
    head, small = _sizes(case)
    # every gradient read, every result written
    return {"bytes": 2 * (4 * sum(head) + size[case["dtype"]] * sum(small)) + 4, "flops": 3 * (sum(head) + sum(small))}


def exact(case, seed):
    """The same from the definitions in 64 bits."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "embed":
        one = torch.cat([s.table.double(), torch.zeros(1, case["d"], dtype=torch.float64, device="cuda")])       # row v: padding
        pick = torch.where(s.tokens < 0, case["v"], s.tokens).long()
        if pick.numel() * case["d"] > 1 << 28:
            return None
        return [torch.index_select(one * s.scale, 0, pick)]
    if op == "embed_grad":
        # running sums over the positions in order of their tokens; a token's sum is the difference at its ends
        sorted_tokens, order = torch.sort(s.tokens.long(), stable=True)
        total = torch.zeros(s.tokens.numel() + 1, case["d"], dtype=torch.float64, device="cuda")
        torch.cumsum(s.d_out[order].double(), 0, out=total[1:])
        ends = torch.searchsorted(sorted_tokens, torch.arange(case["v"] + 1, device="cuda"))
        return [(total[ends[1:]] - total[ends[:-1]]) * s.scale]
    if op == "norm":
        x = s.x.double() + s.residual.double()
        length = torch.sqrt(torch.linalg.vector_norm(x, dim=1) ** 2 / case["d"] + EPS)
        y = torch.einsum("td,t,d->td", x, 1.0 / length, s.weight.double())
        if not case["bits8"]:
            return [x, y]
        scales, codes = [], []
        for part in torch.split(y, case["group"] or case["d"], dim=1):
            scale = part.abs().max(dim=1, keepdim=True).values / 448.0
            scale = scale + (scale == 0)
            scales.append(scale)
            codes.append(_nearest_e4m3(part / scale))
        return [x, torch.cat(codes, 1), torch.cat(scales, 1)]
    if op == "norm_grad":
        x, w, dy = s.x.double(), s.weight.double(), s.d_out.double()
        length = torch.sqrt(torch.linalg.vector_norm(x, dim=1, keepdim=True) ** 2 / case["d"] + EPS)
        unit, up = x / length, dy * w                                  # d out = up . d unit; d unit = (1 - unit unit^T / d) d x / length
        dx = (up - unit * (up * unit).sum(1, keepdim=True) / case["d"]) / length
        return [dx if s.d_sum is None else dx + s.d_sum.double(), torch.einsum("td,td->d", dy, unit)]
    head, small = s.head.double(), s.small.double()
    norm = torch.hypot(torch.linalg.vector_norm(head), torch.linalg.vector_norm(small))
    ratio = min(1.0, case["max_norm"] / float(norm))
    return [norm.reshape(1), head.mul_(ratio), small.mul_(ratio)]


def _nearest_e4m3(x):
    """The nearest value of three mantissa bits (ties to even), steps of 2^-9 below 2^-6, at most 448."""
    _, exponent = torch.frexp(x)
    step = torch.exp2((exponent - 1).clamp_min(-6).double() - 3)
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)
