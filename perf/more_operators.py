"""Fine-tuning around the head, as sized calls: adaptors beside a projection, dropout, and the losses of windows' log-likelihoods.

A model that feeds a head is fitted to several tasks by low-rank adaptors and trained on what its windows are worth:
  project       out[t] = W x[t] + A[i] low[t] with low[t] = scale[i] * B[i] x[t], i the adaptor of row t's request (negative: none). Rows of one
                request follow each other in a prompt or a training batch; in a decoding step every row is another request. With `keep` low is returned
                too, for the gradient
  project_grad  d_x = W^T d_out + B[i]^T v, v[t] = scale[i] * A[i]^T d_out[t]; dA[i] = sum of d_out low^T and dB[i] = sum of v x^T over the rows of i
  dropout       out = residual + (x / (1 - p) where a draw says so, else 0); the draws are 16-bit parts of Philox4x32-10 of (element / 8, step) under a
                seed, so the gradient's call makes the same mask again
  policy        positions t of sequences: ratio = exp(logp - old), loss = -min(ratio * a, clip(ratio, 1 - low, 1 + high) * a) + beta * (exp(q) - q - 1) with
                q = ref - logp, averaged over the valid positions, or over each sequence's and then over the sequences; its gradient in logp, and
                the averages of its first part, of its second and of the clipped positions
  preference    sequences 2p (chosen) and 2p + 1: h = beta * (sum of logp - ref over the chosen one's valid positions - that over the other's); the loss
                is the mean of -(1 - s) log sigmoid(h) - s log sigmoid(-h); its gradient in logp, and every h
Inputs are synthetic: activations ~N(0,1) as a norm leaves them, log-likelihoods as windows of bytes have them and small shifts between the policies.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
_SMALL = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one sequence being decoded with its adaptor
        dict(op="project", name="project_step_1", T=1, d=4096, m=4096, k=16, S=8, packed=False, keep=False),
        # a decoding step of 64 sequences that use 32 adaptors
        dict(op="project", name="project_step_64", T=64, d=4096, m=4096, k=16, S=32, packed=False, keep=False),
        # prompts of eight requests
        dict(op="project", name="project_prompt_8192", T=8192, d=4096, m=4096, k=16, S=8, packed=True, keep=False),
        # an uneven training batch of odd widths, with what its gradient needs
        dict(op="project", name="project_odd_2005", T=2005, d=1001, m=2003, k=12, S=5, packed=True, keep=True),
        # the gradient of a training batch with one adaptor
        dict(op="project_grad", name="project_grad_8192", T=8192, d=4096, m=4096, k=16, S=1, packed=True),
        # of several tasks at once, of higher rank
        dict(op="project_grad", name="project_grad_ragged_2005", T=2005, d=2048, m=4096, k=64, S=6, packed=True),
        # a training batch's activations on their way into the residual stream
        dict(op="dropout", name="dropout_8192", T=8192, d=4096, io="bf16", residual=True, p=0.1),
        # fp32 gradients of an odd width on their way back
        dict(op="dropout", name="dropout_odd_693", T=693, d=1001, io="f32", residual=False, p=0.25),
        # a few short answers
        dict(op="policy", name="policy_512", S=8, most=64, masked=False, by="positions", beta=0.0),
        # a batch of groups of long ones, with prompts masked
        dict(op="policy", name="policy_million", S=256, most=8192, masked=True, by="sequences", beta=0.04),
        # eight pairs of short answers
        dict(op="preference", name="preference_8", S=16, most=128, masked=False, smooth=0.0),
        # a batch of pairs of long ones
        dict(op="preference", name="preference_million", S=256, most=8192, masked=True, smooth=0.1),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(["project", "project", "project_grad", "dropout", "policy", "preference"])
    if op in ("project", "project_grad"):
        d, m = (_log_uniform(rng, 128, 8192) for _ in range(2))
        if rng.random() < 0.75:
            d, m = (d + 15) // 16 * 16, (m + 7) // 8 * 8
        T = min(_log_uniform(rng, 1, 8192), 8192 * 4096 * 4096 // (d * m))
        case = dict(op=op, T=max(1, T), d=d, m=m, k=rng.choice([8, 16, 16, 32, 64, rng.randint(1, 64)]), S=_log_uniform(rng, 1, 64))
        if op == "project_grad":
            return dict(case, S=min(case["S"], 8), packed=True)
        return dict(case, packed=T > 256 or rng.random() < 0.3, keep=rng.random() < 0.3)
    if op == "dropout":
        d = _log_uniform(rng, 64, 8192)
        if rng.random() < 0.75:
            d = (d + 7) // 8 * 8
        return dict(op=op, T=_log_uniform(rng, 1, min(16384, 8192 * 4096 // d)), d=d, io=rng.choice(["bf16", "f32"]), residual=rng.random() < 0.5,
                    p=rng.choice([0.05, 0.1, 0.25, 0.5, round(rng.uniform(0.01, 0.9), 3)]))
    case = dict(op=op, S=2 * _log_uniform(rng, 1, 256), most=_log_uniform(rng, 12, 8192), masked=rng.random() < 0.5)
    case["most"] = max(12, min(case["most"], 256 * 8192 // case["S"]))
    if op == "policy":
        return dict(case, by=rng.choice(["positions", "sequences"]), beta=rng.choice([0.0, 0.01, 0.04]))
    return dict(case, smooth=rng.choice([0.0, 0.0, 0.1, 0.25]))


class _State:
    pass


def _lengths(case):
    """Lengths of a batch's sequences, between half of the longest and all of it."""
    S, most = case["S"], case["most"]
    return [most - (i * 7919 + i * i) % (most // 2 + 1) for i in range(S)]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, dtype=dtype, device="cuda")

    s = _State()
    s.case = case
    op, bf16 = case["op"], torch.bfloat16
    if op in ("project", "project_grad"):
        T, d, m, k, S = (case[c] for c in "TdmkS")
        s.x, s.W = normal(T, d, dtype=bf16), normal(m, d, std=0.02, dtype=bf16)
        s.A, s.B = normal(S, m, k, std=0.02, dtype=bf16), normal(S, k, d, std=d ** -0.5, dtype=bf16)
        s.scale = 1.0 + torch.rand(S, device="cuda", generator=g)
        # every ninth request (or row, where each is another request) has no adaptor
        if case["packed"]:
            request = torch.arange(T, device="cuda") * (S + S // 8 + 1) // max(T, 1)
            order = torch.randperm(S + S // 8 + 1, device="cuda", generator=g)
            which = torch.where(order < S, order, -1)[request] if S > 1 else torch.zeros(T, device="cuda")
        else:
            which = torch.randint(0, S, (T,), device="cuda", generator=g)
            which = torch.where(torch.arange(T, device="cuda") % 9 == 8, -1, which)
        s.which = which.to(torch.int32)
        if op == "project":
            s.out, s.low = empty(T, m, dtype=bf16), empty(T, k) if case["keep"] else None
        else:
            s.d_out = normal(T, m, std=1e-3, dtype=bf16)
            s.low = _low(s.x, s.B, s.scale, s.which)
            s.d_x, s.dA, s.dB = empty(T, d, dtype=bf16), empty(S, m, k), empty(S, k, d)
    elif op == "dropout":
        T, d, io = case["T"], case["d"], _SMALL[case["io"]]
        s.x, s.out = normal(T, d, dtype=io), empty(T, d, dtype=io)
        s.residual = normal(T, d, dtype=io) if case["residual"] else None
        s.rng = torch.tensor([seed * 1000003 + 12345678901, 17 + seed], dtype=torch.int64, device="cuda")        # seed, step
        s.layer = 5                                            # the call's place in its step
    else:
        lengths = torch.tensor(_lengths(case), device="cuda")
        s.offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), lengths.cumsum(0)]).to(torch.int32)
        T, S = sum(_lengths(case)), case["S"]
        s.logp = -11.0 * torch.rand(T, device="cuda", generator=g) - 0.01                      # windows of eight bytes
        s.ref = s.logp + normal(T, std=0.1)
        s.mask = None
        if case["masked"]:                                     # the front of every sequence is its prompt, a few positions are padding
            at = torch.arange(T, device="cuda") - s.offsets[:-1].repeat_interleave(lengths)
            s.mask = (at * 4 >= lengths.repeat_interleave(lengths)) & (torch.rand(T, device="cuda", generator=g) < 0.97)
        s.d_logp, s.loss = empty(T), empty(1)
        if op == "policy":
            s.old = s.logp + normal(T, std=0.15)
            s.advantage = normal(S) + 0.25
            s.stats = empty(3)
        else:
            s.h = empty(S // 2)
    return s


LOW, HIGH, BETA = 0.1875, 0.25, 0.125             # clipping range; inverse temperature of the preference loss


def run(s):
    case, op = s.case, s.case["op"]
    if own:
        from paper_2511_11346_b200 import binding
        if op == "project":
            binding.mtpc_adapted_projection(s.x, s.W, s.A, s.B, s.scale, s.which, s.out, out_low=s.low)
            return [s.out, s.low] if case["keep"] else [s.out]
        if op == "project_grad":
            binding.mtpc_adapted_projection_backward(s.x, s.W, s.A, s.B, s.scale, s.which, s.low, s.d_out, s.d_x, s.dA, s.dB)
            return [s.d_x, s.dA, s.dB]
        if op == "dropout":
            binding.mtpc_dropout(s.x, s.out, case["p"], s.rng, offset=s.layer, residual=s.residual)
            return [s.out]
        if op == "policy":
            binding.mtpc_policy_loss(s.logp, s.old, s.ref if case["beta"] else None, s.advantage, s.offsets, LOW, HIGH, case["beta"], s.loss, s.d_logp,
                                     mask=s.mask, by_sequence=case["by"] == "sequences", out_stats=s.stats)
            return [s.loss, s.d_logp, s.stats]
        binding.mtpc_preference_loss(s.logp, s.ref, s.offsets, BETA, s.loss, s.d_logp, mask=s.mask, smoothing=case["smooth"], out_h=s.h)
        return [s.loss, s.d_logp, s.h]

    if op == "project":
        low = _low(s.x, s.B, s.scale, s.which)
        out = s.x.float() @ s.W.float().T + _spread(low, s.which, case["S"]) @ s.A.float().transpose(1, 2).reshape(-1, case["m"])
        return [out.to(s.x.dtype), low] if case["keep"] else [out.to(s.x.dtype)]
    if op == "project_grad":
        T, d, m, k, S = (case[c] for c in "TdmkS")
        d_out = s.d_out.float()
        v = _low(s.d_out, s.A.transpose(1, 2), s.scale, s.which)
        v_all, low_all = _spread(v, s.which, S), _spread(s.low, s.which, S)
        d_x = d_out @ s.W.float() + v_all @ s.B.float().reshape(S * k, d)
        return [d_x.to(s.x.dtype), (low_all.T @ d_out).view(S, k, m).transpose(1, 2).contiguous(), (v_all.T @ s.x.float()).view(S, k, d)]
    if op == "dropout":
        cut = _cut(case["p"])
        kept = _draws(s.x.numel(), s.rng, s.layer).view(s.x.shape) >= cut
        y = torch.where(kept, s.x.float() * (65536.0 / (65536 - cut)), 0.0)
        return [(y if s.residual is None else y + s.residual.float()).to(s.x.dtype)]
    lengths = (s.offsets[1:] - s.offsets[:-1]).long()
    of = torch.repeat_interleave(torch.arange(case["S"], device="cuda"), lengths)
    valid = torch.ones_like(s.logp, dtype=torch.bool) if s.mask is None else s.mask
    logp, S = s.logp.double(), case["S"]
    if op == "policy":
        ratio = torch.exp(logp - s.old.double())
        a = s.advantage.double()[of]
        held = ratio.clamp(1.0 - LOW, 1.0 + HIGH) * a
        clipped = held < ratio * a
        count = torch.zeros(S, dtype=torch.float64, device="cuda").index_add_(0, of, valid.double())
        share = 1.0 / (S * count.clamp_min(1.0))[of] if case["by"] == "sequences" else 1.0 / count.sum().clamp_min(1.0)
        share = torch.where(valid, share, 0.0)
        q = (s.ref.double() - logp) * (1.0 if case["beta"] else 0.0)
        kl = torch.exp(q) - q - 1.0
        grad = torch.where(clipped, 0.0, -ratio * a) + case["beta"] * (1.0 - torch.exp(q))
        stats = torch.stack([(share * -torch.minimum(held, ratio * a)).sum(), (share * kl).sum(), (share * clipped).sum()])
        return [(stats[0] + case["beta"] * stats[1]).float().reshape(1), (share * grad).float(), stats.float()]
    sums = torch.zeros(S, dtype=torch.float64, device="cuda").index_add_(0, of, torch.where(valid, logp - s.ref.double(), 0.0))
    h, smooth = BETA * (sums[0::2] - sums[1::2]), case["smooth"]
    loss = ((1.0 - smooth) * torch.log1p(torch.exp(-h.abs())) + smooth * torch.log1p(torch.exp(-h.abs()))
            + (1.0 - smooth) * (-h).clamp_min(0.0) + smooth * h.clamp_min(0.0)).mean()
    slope = BETA * (smooth - (1.0 / (1.0 + torch.exp(h)))) / len(h)
    d_logp = torch.where(valid, torch.stack([slope, -slope], 1).flatten()[of], 0.0)
    return [loss.float().reshape(1), d_logp.float(), h.float()]


def _low(x, B, scale, which):
    """scale[i] * B[i] x[t], i = which[t]; zeros where that is negative."""
    S, k = B.shape[0], B.shape[1]
    every = (x.float() @ B.float().reshape(S * k, -1).T).view(-1, S, k)
    i = which.clamp_min(0).long()
    low = torch.take_along_dim(every, i[:, None, None], 1)[:, 0] * scale[i][:, None]
    return torch.where(which[:, None] < 0, 0.0, low)


def _spread(low, which, S):
    """[T, k] -> [T, S k] with each row in its adaptor's columns."""
    mine = which[:, None] == torch.arange(S, device="cuda")
    return (mine[:, :, None] * low[:, None, :]).flatten(1)


def _cut(p):
    """Draws below this one drop: p in steps of 2^-16."""
    return min(65535, int(math.floor(p * 65536.0 + 0.5)))


def _draws(count, rng, layer):
    """Sixteen-bit draws: element e has part e % 8 of the block e // 8, parts of a word from its lower half on."""
    low32 = 0xFFFFFFFF

    def times(a, b):                                           # the 64-bit product's halves, of a constant and a tensor of 32-bit values
        p, q = (a & 0xFFFF) * b, (a >> 16) * b
        return (q + (p >> 16)) >> 16, (((q & 0xFFFF) << 16) + p) & low32
    block = torch.arange((count + 7) // 8, device="cuda")
    step = rng[1] + layer
    c = [block & low32, block >> 32, (step & low32).expand_as(block), ((step >> 32) & low32).expand_as(block)]
    key = [rng[0] & low32, (rng[0] >> 32) & low32]
    for _ in range(10):
        (h0, l0), (h1, l1) = times(0xD2511F53, c[0]), times(0xCD9E8D57, c[2])
        c = [h1 ^ c[1] ^ key[0], l1, h0 ^ c[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) & low32, (key[1] + 0xBB67AE85) & low32]
    words = torch.stack(c, 1)
    return torch.stack([words & 0xFFFF, words >> 16], 2).flatten()[:count]


def work(case):
    op = case["op"]
    if op in ("project", "project_grad"):
        T, d, m, k, S = (case[c] for c in "TdmkS")
        used = min(S, T)
        params = 2 * (m * d + used * k * (d + m)) + 8 * T
        if op == "project":
            return {"bytes": params + 2 * T * (d + m) + (4 * T * k if case["keep"] else 0), "flops": 2 * T * (d * m + k * (d + m))}
        # x, d_out and low read, d_x and all of dA and dB written
        return {"bytes": params + 2 * T * (2 * d + m) + 4 * T * k + 4 * S * k * (d + m), "flops": 2 * T * (d * m + 2 * k * (d + m))}
    if op == "dropout":
        n, b = case["T"] * case["d"], 2 if case["io"] == "bf16" else 4
        return {"bytes": n * b * (3 if case["residual"] else 2), "flops": 2 * n}
    T, S = sum(_lengths(case)), case["S"]
    read = (12 if case["beta"] else 8) if op == "policy" else 8
    return {"bytes": T * (read + 4 + (1 if case["masked"] else 0)) + 12 * S, "flops": T * (20 if op == "policy" else 3)}


def exact(case, seed):
    """The same from the definitions in 64 bits."""
    s = prepare(case, seed)
    op = case["op"]
    if op in ("project", "project_grad"):
        S, rows = case["S"], [torch.nonzero(s.which == i).flatten() for i in range(case["S"])]
        x = s.x.double()
        if op == "project":
            out = torch.mm(x, s.W.double().t())
            low = torch.zeros(case["T"], case["k"], dtype=torch.float64, device="cuda")
            for i in range(S):
                low[rows[i]] = float(s.scale[i]) * torch.mm(x[rows[i]], s.B[i].double().t())
                out[rows[i]] += torch.mm(low[rows[i]], s.A[i].double().t())
            return [out, low] if case["keep"] else [out]
        d_out, low = s.d_out.double(), s.low.double()
        d_x = torch.mm(d_out, s.W.double())
        dA, dB = torch.zeros_like(s.dA, dtype=torch.float64), torch.zeros_like(s.dB, dtype=torch.float64)
        for i in range(S):
            dy = d_out[rows[i]]
            v = torch.mm(dy, s.A[i].double()) * float(s.scale[i])
            d_x[rows[i]] += torch.mm(v, s.B[i].double())
            dA[i], dB[i] = torch.mm(dy.t(), low[rows[i]]), torch.mm(v.t(), x[rows[i]])
        return [d_x, dA, dB]
    if op == "dropout":
        n = s.x.numel()
        seed_, step = (int(w) for w in s.rng.tolist())
        kept = torch.from_numpy(_philox(n, seed_, step + s.layer) >= _cut(case["p"])).cuda().view(s.x.shape)
        y = s.x.double() / (1.0 - _cut(case["p"]) / 65536.0) * kept
        return [y if s.residual is None else s.residual.double() + y]
    starts = s.offsets.tolist()
    valid = torch.ones(len(s.logp), dtype=torch.bool, device="cuda") if s.mask is None else s.mask
    logp, d_logp = s.logp.double(), torch.zeros(len(s.logp), dtype=torch.float64, device="cuda")
    if op == "policy":
        total = max(1, int(valid.sum()))
        stats = torch.zeros(3, dtype=torch.float64, device="cuda")
        for i, (b, e) in enumerate(zip(starts, starts[1:])):
            ok = torch.nonzero(valid[b:e]).flatten() + b
            part = 1.0 / (case["S"] * max(1, len(ok))) if case["by"] == "sequences" else 1.0 / total
            r, a = torch.exp(logp[ok] - s.old.double()[ok]), s.advantage.double()[i]
            # a gain beyond the upper end, or a loss beyond the lower one, counts as the end's
            out = (a > 0) & (r > 1.0 + HIGH) | (a < 0) & (r < 1.0 - LOW)
            value = torch.where(out, torch.where(a > 0, 1.0 + HIGH, 1.0 - LOW), r) * a
            stats[0] -= part * value.sum()
            stats[2] += part * out.sum()
            slope = -torch.where(out, 0.0, r) * a
            if case["beta"]:
                q = s.ref.double()[ok] - logp[ok]
                stats[1] += part * (torch.expm1(q) - q).sum()
                slope = slope - case["beta"] * torch.expm1(q)
            d_logp[ok] = part * slope
        return [(stats[0] + case["beta"] * stats[1]).reshape(1), d_logp, stats]
    ratio = torch.where(valid, logp - s.ref.double(), 0.0)
    sums = torch.stack([ratio[b:e].sum() for b, e in zip(starts, starts[1:])]).view(-1, 2)
    h, e = BETA * (sums[:, 0] - sums[:, 1]), case["smooth"]
    logsigmoid = torch.nn.functional.logsigmoid
    loss = -((1 - e) * logsigmoid(h) + e * logsigmoid(-h)).mean()
    slope = -BETA * ((1 - e) * torch.sigmoid(-h) - e * torch.sigmoid(h)) / len(h)
    for p, g in enumerate(slope.tolist()):
        d_logp[starts[2 * p]:starts[2 * p + 1]] = g
        d_logp[starts[2 * p + 1]:starts[2 * p + 2]] = -g
    return [loss.reshape(1), d_logp * valid, h]


def _philox(count, seed, step):
    """The sixteen-bit draws by numpy's wrapping 64-bit products."""
    u = np.uint64
    half, word = u(32), u(0xFFFFFFFF)
    block = np.arange(-(-count // 8), dtype=u)
    x0, x1 = block & word, block >> half
    x2, x3 = np.full_like(block, step & 0xFFFFFFFF), np.full_like(block, step >> 32 & 0xFFFFFFFF)
    for i in range(10):
        k0, k1 = u((seed + i * 0x9E3779B9) & 0xFFFFFFFF), u(((seed >> 32) + i * 0xBB67AE85) & 0xFFFFFFFF)
        a, b = x0 * u(0xD2511F53), x2 * u(0xCD9E8D57)
        x0, x1, x2, x3 = (b >> half) ^ x1 ^ k0, b & word, (a >> half) ^ x3 ^ k1, a & word
    out = np.empty((len(block), 4, 2), dtype=np.int64)
    for i, x in enumerate((x0, x1, x2, x3)):
        out[:, i, 0], out[:, i, 1] = x & u(0xFFFF), x >> u(16)
    return out.reshape(-1)[:count]
