"""The token operators beside the verifier: what a program computes from a model's logits before and
after the library has looked at its answers.

  score      log probabilities of given tokens, entropy and the best alternatives, over the
             tokens a decoding mask leaves (vl_token_logprobs)
  grad       their gradient in the logits (vl_token_logprobs_grad)
  advantage  counted violations -> rewards -> advantages within each program's samples
             (vl_group_advantages)
  policy     the clipped policy loss of the samples and its gradient in the tokens' log
             probabilities (vl_policy_loss)

A sample is one register per operand occurrence, so a token stands for a register where the
vocabulary is a window of 512, the library's largest register file; wider rows are scored over a
model's whole vocabulary.  Sample lengths are those of the benchmark's programs (2.6-2.9
occurrences per instruction, 200-20,000 instructions), K = 100 or 1,000 samples each.

With `own` false the operators are computed in their plain form, in torch's elementary
operations; with `own` true by the library.
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
NO = float("-inf")


def listed():
    def rows(name, op, n_row, n_vocab, type, **more):
        return {"name": name, "op": op, "rows": n_row, "vocab": n_vocab, "type": type, "first": 0, "pitch": 0, "mask": False,
                "given": True, "entropy": False, "top": 0, "scale": 1.0, "padded": 0.0, **more}

    def policy(name, n_program, k, n_occ, **more):
        return {"name": name, "op": "policy", "programs": n_program, "k": k, "occ": n_occ, "layout": "rows", "ref": False,
                "stopped": 0.0, "kl": 0.0, **more}
    return [
        # one decoding step of one program's 100 samples: the registers' window of the vocabulary under the
        # decoding mask, the eight best to choose from; latency counts
        rows("score_step_100x512", "score", 100, 512, "bf16", first=32000, pitch=32512, mask=True, given=False, top=8),
        # one step of one request over a whole vocabulary, with the usual twenty alternatives
        rows("score_next_1x131072", "score", 1, 131072, "bf16", given=False, entropy=True, top=20),
        # one emitted register of each of 256 programs' 100 samples scored for training, a tenth already ended
        rows("score_sweep_25600x512", "score", 25600, 512, "bf16", mask=True, entropy=True, padded=0.1),
        # whole sequences scored over a vocabulary of odd size, with a short list of alternatives
        rows("score_seq_4096x50001", "score", 4096, 50001, "f16", entropy=True, top=5),
        # constrained scoring in 32 bits under a mask over the whole vocabulary, a temperature
        rows("score_mask_500x32000", "score", 500, 32000, "f32", mask=True, entropy=True, top=1, scale=1.4),
        # the gradients of a training step: registers under the mask with an entropy bonus, sequences in 32 bits over an odd
        # vocabulary, and the largest, over a large vocabulary
        rows("grad_sweep_25600x512", "grad", 25600, 512, "bf16", mask=True, entropy=True, padded=0.1),
        rows("grad_seq_1024x50001", "grad", 1024, 50001, "f32", scale=0.7),
        rows("grad_large_8192x131072", "grad", 8192, 131072, "bf16", padded=0.05),
        # advantages of one program's samples, and of a whole sweep with many samples each
        {"name": "advantage_1x100", "op": "advantage", "programs": 1, "k": 100, "extra": False},
        {"name": "advantage_256x1000", "op": "advantage", "programs": 256, "k": 1000, "extra": True},
        # the loss over one loop kernel's samples against a reference model, and over 16 large kernels' of up to 20,000 instructions
        policy("policy_loop_1x100", 1, 100, 5261, ref=True, kl=0.05, stopped=0.2),
        policy("policy_mha_16x100", 16, 100, 56800, layout="packed", stopped=0.1),
    ]


def draw(rng):
    """One more case of the ranges above; sizes on a logarithmic scale."""
    def spread(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    op = rng.choice(["score", "score", "score", "grad", "grad", "grad", "advantage", "policy", "policy"])
    if op == "advantage":
        return {"op": op, "programs": spread(1, 256), "k": spread(1, 1000), "extra": rng.random() < 0.5}
    if op == "policy":
        occ = spread(1, 57000)
        k = spread(1, 1000)
        n = max(1, min(spread(1, 256), int(9e7 / (occ * k))))
        k = max(1, min(k, int(9e7 / (occ * n))))
        ref = rng.random() < 0.5
        return {"op": op, "programs": n, "k": k, "occ": occ, "layout": rng.choice(["rows", "packed"]), "ref": ref,
                "stopped": rng.choice([0.0, 0.1, 0.5]), "kl": 0.05 if ref else 0.0}
    vocab = rng.choice([512, 512, spread(2, 4096), spread(4096, 131072), spread(2, 131072)])
    n = max(1, min(spread(1, 25600), int((2e8 if op == "score" else 4e8) / vocab)))
    given = op == "grad" or rng.random() < 0.6
    top = rng.choice([0, 1, 5, 8, 20, 32]) if op == "score" else 0
    case = {"op": op, "rows": n, "vocab": vocab, "type": rng.choice(["bf16", "bf16", "f16", "f32"]),
            "first": rng.choice([0, 0, rng.randint(1, 300)]), "pitch": 0, "mask": rng.random() < 0.5, "given": given,
            "entropy": rng.random() < 0.6 or (not given and not top), "top": top, "scale": rng.choice([1.0, 1.0, 0.7, 1.4]),
            "padded": rng.choice([0.0, 0.0, 0.2]) if given else 0.0}
    if case["first"] or rng.random() < 0.3:
        case["pitch"] = case["first"] + vocab + rng.randint(0, 64)
    return case


# ---- inputs

def _logits(case, gen):
    """Rows of a trained model's logits: a bell with a few tokens far above it, and in whole vocabularies a tail of
    ids that no token has, filled with the type's lowest value."""
    n, v, dtype = case["rows"], case["vocab"], TYPES[case["type"]]
    pitch = case["pitch"] or v
    x = torch.empty((n, pitch), dtype=dtype, device="cuda")
    for r in range(0, n, 1024):
        x[r:r + 1024] = (torch.randn((min(1024, n - r), pitch), generator=gen, device="cuda") * 2).to(dtype)
    x = x[:, case["first"]:case["first"] + v]
    few = min(4, v)   # distinct ones
    likely = (torch.randint(0, v, (n, 1), generator=gen, device="cuda") + torch.arange(few, device="cuda") * (v // few)) % v
    x.scatter_add_(1, likely, (torch.rand((n, few), generator=gen, device="cuda") * 4 + 5).to(dtype))
    if v > 4096:
        x[:, v - 7:] = torch.finfo(dtype).min
    return x, likely


def _rows(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n, v = case["rows"], case["vocab"]
    x, likely = _logits(case, gen)
    s = {"logits": x, "token": None, "mask": None}
    # a sampled token: mostly a likely one
    other = torch.randint(0, v, (n,), generator=gen, device="cuda")
    token = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.7, likely[:, 0], other)
    if case["mask"]:
        words = (v + 31) // 32

        def bits():
            return torch.randint(-2 ** 31, 2 ** 31, (n, words), generator=gen, device="cuda")
        m = bits() | (bits() & bits())   # five in eight registers are free
        m[torch.rand(n, generator=gen, device="cuda") < 0.01] = 0   # no register is free: the sample has failed
        if case["given"]:
            at = (token >> 5)[:, None]
            m.scatter_(1, at, m.gather(1, at) | (1 << (token & 31))[:, None])
        s["mask"] = ((m + 2 ** 31) % 2 ** 32 - 2 ** 31).to(torch.int32)
    if case["given"]:
        ended = torch.rand(n, generator=gen, device="cuda") < case["padded"]
        s["token"] = torch.where(ended, -1, token).to(torch.int32)
    if case["op"] == "grad":
        s["g_logprob"] = torch.randn(n, generator=gen, device="cuda") / n
        s["g_entropy"] = -torch.rand(n, generator=gen, device="cuda") * 0.1 / n if case["entropy"] else None
    return s


def _lengths(case, gen):
    """Where each sample's tokens start and how many there are: rows of one pitch per program, or packed; a share
    of the samples was stopped early, some before their first token."""
    n, k, occ = case["programs"], case["k"], case["occ"]
    sizes = random.Random(n * 100003 + occ)   # (a program's length is the case's, not the seed's)
    own_occ = torch.tensor([occ] + [sizes.randint((occ + 1) // 2, occ) for _ in range(n - 1)], device="cuda")
    pitch = (own_occ + 63) // 64 * 64 if case["layout"] == "rows" else own_occ
    room, full = pitch.repeat_interleave(k), own_occ.repeat_interleave(k)
    start = room.cumsum(0) - room
    cut = (torch.rand(n * k, generator=gen, device="cuda") * (full + 1)).long().minimum(full)
    length = torch.where(torch.rand(n * k, generator=gen, device="cuda") < case["stopped"], cut, full)
    return start, length, int(room.sum()), int(length.sum())


def _policy(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    start, length, size, count = _lengths(case, gen)
    n = start.numel()
    logprob = torch.rand(size, generator=gen, device="cuda").square_().add_(1e-6).log_()
    s = {"start": start, "length": length.to(torch.int32), "tokens": count, "logprob": logprob, "ref": None,
         "old": logprob + torch.randn(size, generator=gen, device="cuda").mul_(0.15)}
    if case["ref"]:
        s["ref"] = logprob + torch.randn(size, generator=gen, device="cuda").mul_(0.2)
    s["advantage"] = torch.randn(n, generator=gen, device="cuda")
    s["advantage"][torch.rand(n, generator=gen, device="cuda") < 0.05] = 0.0
    s["weight"] = torch.full((n,), 1.0 / max(1, count), device="cuda")
    s["grad"] = torch.zeros(size, device="cuda")
    return s


def _counts(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = case["programs"] * case["k"]
    c = torch.zeros((n, 8), dtype=torch.int32, device="cuda")
    for word, share, most in ((1, 0.3, 40), (2, 0.1, 5), (3, 0.25, 2000)):
        some = torch.rand(n, generator=gen, device="cuda") < share
        c[:, word] = torch.where(some, torch.randint(1, most, (n,), generator=gen, device="cuda"), 0).to(torch.int32)
    c[:, 0] = (c[:, 1] > 0).int() | (c[:, 2] > 0).int() << 1 | (c[:, 3] > 0).int() << 2
    c[:, 4] = (c[:, 2] > 0).int()
    s = {"counts": c, "weights": (1.0, -0.02, -0.1, -0.003), "eps": 1e-6, "extra": None}
    s["offsets"] = torch.arange(0, n + 1, case["k"], dtype=torch.int32, device="cuda")
    if case["extra"]:
        s["extra"] = -0.001 * torch.randint(0, 500, (n,), generator=gen, device="cuda").float()
    return s


def prepare(case, seed):
    op = case["op"]
    if op == "policy":
        s = _policy(case, seed)
        s["stats"] = torch.zeros(24, dtype=torch.uint8, device="cuda")
        s["log_lo"], s["log_hi"] = -0.21875, 0.25   # ratios from 0.80 to 1.28, bounds that 32 bits hold exactly
    elif op == "advantage":
        s = _counts(case, seed)
        n = s["counts"].shape[0]
        s["advantage"], s["reward"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    else:
        s = _rows(case, seed)
        n = case["rows"]
        if op == "score":
            s["logprob"] = torch.empty(n, device="cuda") if case["given"] else None
            s["entropy"] = torch.empty(n, device="cuda") if case["entropy"] else None
            s["stat"] = torch.empty((n, 2), device="cuda") if case["given"] else None
            s["top_token"] = torch.empty((n, case["top"]), dtype=torch.int32, device="cuda") if case["top"] else None
            s["top_logprob"] = torch.empty((n, case["top"]), device="cuda") if case["top"] else None
        else:   # what the forward pass left
            parts = [_plain_stats(s["logits"][r:r + 1024], None if s["mask"] is None else s["mask"][r:r + 1024], case["scale"], 64)
                     for r in range(0, n, 1024)]
            top, log_sum, entropy = (torch.cat(p).float() for p in zip(*parts))
            ended = s["token"] < 0
            s["stat"] = torch.stack([top, log_sum], 1).masked_fill(ended[:, None], 0.0)
            s["entropy"] = entropy.masked_fill(ended, 0.0) if case["entropy"] else None
            s["grad"] = torch.empty((n, case["vocab"]), dtype=s["logits"].dtype, device="cuda")
    s["case"] = case
    return s


# ---- the plain forms

def _allowed(logits, mask):
    """[rows, tokens] or None"""
    if mask is None:
        return None
    t = torch.arange(logits.shape[1], device=logits.device)
    return (mask[:, t >> 5] >> (t & 31).int()) & 1 == 1


def _plain_rows(logits, mask, scale, width):
    """(largest logit, scaled distance of each logit to it), in 32 or 64 bits"""
    x = logits.double() if width == 64 else logits.float()
    allowed = _allowed(x, mask)
    if allowed is not None:
        x = x.masked_fill(~allowed, NO)
    top = x.amax(1)
    return x, top, (x - torch.where(top == NO, 0.0, top)[:, None]) * scale


def _plain_stats(logits, mask, scale, width):
    """(largest logit, log of the sum, entropy)"""
    x, top, z = _plain_rows(logits, mask, scale, width)
    e = z.exp()
    total = e.sum(1)
    log_sum = total.log()
    mean = (e * torch.where(e > 0, z, 0.0)).sum(1) / total
    return top, log_sum, torch.where(top == NO, 0.0, log_sum - mean)


def _plain_score(s):
    case, token = s["case"], s["token"]
    x, top, z = _plain_rows(s["logits"], s["mask"], case["scale"], 32)
    e = z.exp()
    total = e.sum(1)
    log_sum = total.log()
    nothing = top == NO
    ended = token < 0 if token is not None else torch.zeros_like(nothing)
    out = {}
    if token is not None:
        lp = z.gather(1, token.clamp(min=0).long()[:, None])[:, 0] - log_sum
        out["logprob"] = torch.where(nothing, NO, lp).masked_fill(ended, 0.0)
        out["stat"] = torch.stack([top, log_sum], 1).masked_fill(ended[:, None], 0.0)
    if case["entropy"]:
        mean = (e * torch.where(e > 0, z, 0.0)).sum(1) / total
        out["entropy"] = torch.where(nothing | ended, 0.0, log_sum - mean)
    if case["top"]:
        # by value, equal ones by index: the value's bits as an ordered number above the index's
        k = min(case["top"], x.shape[1])
        bits = (x + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = (order << 32) + (0xFFFFFFFF - torch.arange(x.shape[1], device=x.device))
        best = 0xFFFFFFFF - (key.topk(k, 1).values & 0xFFFFFFFF)
        lp = z.gather(1, best) - log_sum[:, None]
        none = (x.gather(1, best) == NO) | ended[:, None]
        pad = (0, case["top"] - k)
        out["top_token"] = torch.nn.functional.pad(best.int().masked_fill(none, -1), pad, value=-1)
        out["top_logprob"] = torch.nn.functional.pad(lp.masked_fill(none, NO), pad, value=NO)
    return out


def _plain_grad(s):
    case, token, logits = s["case"], s["token"], s["logits"]
    x = logits.float()
    top, log_sum = s["stat"][:, 0], s["stat"][:, 1]
    idle = (token < 0) | (top == NO)
    lp = (x - torch.where(idle, 0.0, top)[:, None]) * case["scale"] - torch.where(idle, 0.0, log_sum)[:, None]
    allowed = _allowed(x, s["mask"])
    if allowed is not None:
        lp = lp.masked_fill(~allowed, NO)
    lp = lp.masked_fill(idle[:, None], NO)
    p = lp.exp()
    g = s["g_logprob"][:, None]
    dx = -g * p
    if s["g_entropy"] is not None:
        dx = dx - s["g_entropy"][:, None] * p * (torch.where(p > 0, lp, 0.0) + s["entropy"][:, None])
    at = token.clamp(min=0).long()[:, None]
    dx = dx.scatter_add(1, at, g.masked_fill(idle[:, None], 0.0))
    if allowed is not None:
        dx = dx.masked_fill(~allowed, 0.0)
    return {"grad": (dx * case["scale"]).to(logits.dtype)}


def _plain_advantage(s):
    c, w = s["counts"], s["weights"]
    r = (c[:, 0] == 0).double() * w[0] + c[:, 1].double() * w[1] + c[:, 2].double() * w[2] + c[:, 3].double() * w[3]
    if s["extra"] is not None:
        r = r + s["extra"].double()
    k = s["case"]["k"]
    g = r.view(-1, k)
    a = (g - g.mean(1, keepdim=True)) / (g.var(1, keepdim=True, unbiased=False).sqrt() + s["eps"])
    return {"reward": r.float(), "advantage": a.reshape(-1).float()}


def _plain_policy(s):
    n, kl = s["start"].numel(), s["case"]["kl"]
    length = s["length"].long()
    sample = torch.arange(n, device="cuda").repeat_interleave(length, output_size=s["tokens"])
    at = torch.arange(s["tokens"], device="cuda") + (s["start"] - (length.cumsum(0) - length))[sample]
    a, w = s["advantage"][sample], s["weight"][sample]
    lp = s["logprob"][at]
    d = lp.double() - s["old"][at].double()   # (in 64 bits: which side of a bound it is on)
    clipped = ((a > 0) & (d > s["log_hi"])) | ((a < 0) & (d < s["log_lo"]))
    ratio = torch.where(clipped, torch.where(a > 0, s["log_hi"], s["log_lo"]), d.float()).exp()
    loss = -a * ratio
    dx = torch.where(clipped, 0.0, loss)
    kls = torch.zeros((), device="cuda", dtype=torch.float64)
    if s["ref"] is not None:
        q = s["ref"][at] - lp
        gap = q.double().expm1() - q.double()
        kls = (w * gap).sum()
        loss = loss + kl * gap
        dx = dx - kl * q.expm1()
    grad = torch.zeros_like(s["logprob"])
    grad[at] = w * dx
    return {"grad": grad, "loss": (w * loss).double().sum().float(), "kl": kls.float(), "tokens": length.sum(), "clipped": clipped.sum()}


# ---- the library's calls

def _own(s):
    import paper_2506_17506_amd as vl
    case = s["case"]
    if case["op"] == "score":
        vl.vl_token_logprobs(s["logits"], token=s["token"], mask=s["mask"], scale=case["scale"], logprob=s["logprob"], entropy=s["entropy"],
                             stat=s["stat"], top_token=s["top_token"], top_logprob=s["top_logprob"])
        return {k: s[k] for k in ("logprob", "stat", "entropy", "top_token", "top_logprob") if s[k] is not None}
    if case["op"] == "grad":
        vl.vl_token_logprobs_grad(s["logits"], s["stat"], s["grad"], token=s["token"], mask=s["mask"], scale=case["scale"],
                                  entropy=s["entropy"], g_logprob=s["g_logprob"], g_entropy=s["g_entropy"])
        return {"grad": s["grad"]}
    if case["op"] == "advantage":
        vl.vl_group_advantages(s["counts"], s["offsets"], s["weights"], s["eps"], s["advantage"], reward=s["reward"], extra=s["extra"])
        return {"reward": s["reward"], "advantage": s["advantage"]}
    vl.vl_policy_loss(s["logprob"], s["old"], s["start"], s["length"], s["advantage"], s["weight"], s["grad"], s["stats"],
                      log_lo=s["log_lo"], log_hi=s["log_hi"], logprob_ref=s["ref"], kl=case["kl"])
    numbers, counts = s["stats"][:8].view(torch.float32), s["stats"][8:].view(torch.int64)
    return {"grad": s["grad"], "loss": numbers[0], "kl": numbers[1], "tokens": counts[0], "clipped": counts[1]}


def run(state):
    if own:
        return _own(state)
    return {"score": _plain_score, "grad": _plain_grad, "advantage": _plain_advantage, "policy": _plain_policy}[state["case"]["op"]](state)


# ---- what a pass cannot do without

def work(case):
    if case["op"] == "advantage":
        n = case["programs"] * case["k"]
        return {"bytes": n * (32 + 8 + 4 * case["extra"]) + 4 * (case["programs"] + 1), "flops": n * 16}
    if case["op"] == "policy":
        n = case["programs"] * case["k"]
        # on average: the first program's samples are the longest, the others' half as long or longer; a stopped one has half its tokens
        count = int(case["k"] * case["occ"] * (0.25 + 0.75 * case["programs"]) * (1.0 - 0.5 * case["stopped"]))
        return {"bytes": count * (12 + 4 * case["ref"]) + n * 20 + 24, "flops": count * (10 + 8 * case["ref"])}
    n, v = case["rows"], case["vocab"]
    live = 1.0 - case["padded"]
    size = 4 if case["type"] == "f32" else 2
    read = live * n * (v * size + (v + 31) // 32 * 4 * case["mask"])
    if case["op"] == "score":
        side = n * (16 * case["given"] + 4 * case["entropy"] + 8 * case["top"])
        return {"bytes": int(read + side), "flops": int(live * n * v * (4 + 2 * case["entropy"]))}
    return {"bytes": int(read + n * v * size + n * (16 + 8 * case["entropy"])), "flops": int(live * n * v * (5 + 3 * case["entropy"]))}


# ---- from the definitions, in 64 bits

def _masked(case, s, r, step):
    """log of the allowed tokens' probabilities of `step` rows, and the allowed logits"""
    x = s["logits"][r:r + step].double()
    if s["mask"] is not None:
        m = s["mask"][r:r + step].long()
        bits = (m[:, :, None] >> torch.arange(32, device="cuda")) & 1
        x = torch.where(bits.flatten(1)[:, :x.shape[1]] == 1, x, NO)
    return torch.log_softmax(x * case["scale"], 1), x


def _exact_rows(case, seed):
    s = _rows(case, seed)
    n, v, step = case["rows"], case["vocab"], max(1, 2 ** 26 // case["vocab"])
    out = {}

    def add(name, value):
        out.setdefault(name, []).append(value)
    for r in range(0, n, step):
        lp, x = _masked(case, s, r, step)
        token = None if s["token"] is None else s["token"][r:r + step].long()
        ended = torch.zeros(len(x), dtype=torch.bool, device="cuda") if token is None else token < 0
        nothing = (x == NO).all(1)
        p = lp.exp()
        h = -torch.special.xlogy(p, p).sum(1)
        if case["op"] == "grad":
            lp, p = lp.masked_fill(nothing[:, None], 0.0), p.masked_fill(nothing[:, None], 0.0)
            here = torch.arange(v, device="cuda") == token[:, None]
            dx = s["g_logprob"][r:r + step].double()[:, None] * (here.double() - p)
            if case["entropy"]:
                inner = torch.special.xlogy(p, p) + p * h.masked_fill(nothing, 0.0)[:, None]
                dx = dx - s["g_entropy"][r:r + step].double()[:, None] * inner
            dx = dx.masked_fill((ended | nothing)[:, None] | (x == NO), 0.0)
            add("grad", dx * case["scale"])
            continue
        if token is not None:
            add("logprob", lp.gather(1, token.clamp(min=0)[:, None])[:, 0].masked_fill(nothing, NO).masked_fill(ended, 0.0))
            top = x.max(1).values
            log_sum = (torch.logsumexp(x * case["scale"], 1) - top * case["scale"]).masked_fill(nothing, NO)
            add("stat", torch.stack([top, log_sum], 1).masked_fill(ended[:, None], 0.0))
        if case["entropy"]:
            add("entropy", h.masked_fill(nothing | ended, 0.0))
        if case["top"]:
            k = min(case["top"], v)
            best = x.topk(k, 1)
            lq = lp.gather(1, best.indices).masked_fill((best.values == NO) | ended[:, None], NO)
            add("top_logprob", torch.cat([lq, torch.full((len(x), case["top"] - k), NO, device="cuda", dtype=torch.float64)], 1))
    out = {name: torch.cat(parts) for name, parts in out.items()}
    if case["top"]:
        out["top_token"] = None
    return out


def _exact_policy(case, seed):
    s = prepare(case, seed)
    inside = torch.zeros(s["logprob"].numel() + 1, dtype=torch.int32, device="cuda")
    some = s["length"] > 0   # (a sample without tokens marks nothing)
    sample = torch.zeros_like(inside)
    first, last = s["start"][some], s["start"][some] + s["length"][some]
    inside.index_add_(0, first, torch.ones_like(first, dtype=torch.int32))
    inside.index_add_(0, last, -torch.ones_like(last, dtype=torch.int32))
    inside = inside.cumsum(0)[:-1] > 0
    ids = torch.arange(len(some), device="cuda", dtype=torch.int32)[some]
    sample.index_add_(0, first, torch.diff(ids, prepend=ids.new_zeros(1)))
    sample = sample.cumsum(0)[:-1]
    a, w = s["advantage"].double()[sample], s["weight"].double()[sample]
    lp = s["logprob"].double()
    ratio = (lp - s["old"].double()).exp()
    near = ratio.clamp(math.exp(s["log_lo"]), math.exp(s["log_hi"]))
    gain = torch.minimum(ratio * a, near * a)
    dx = torch.where(gain == ratio * a, -ratio * a, 0.0)
    loss, kls = -gain, torch.zeros((), dtype=torch.float64, device="cuda")
    if s["ref"] is not None:
        q = s["ref"].double() - lp
        gap = torch.special.expm1(q) - q
        kls = torch.where(inside, w * gap, 0.0).sum()
        loss, dx = loss + case["kl"] * gap, dx - case["kl"] * torch.special.expm1(q)
    return {"grad": torch.where(inside, w * dx, 0.0), "loss": torch.where(inside, w * loss, 0.0).sum(), "kl": kls, "tokens": None, "clipped": None}


def _exact_advantage(case, seed):
    s = _counts(case, seed)
    words = s["counts"].cpu().numpy().astype("f8")
    r = (words[:, 0] == 0) * s["weights"][0] + words[:, 1:4] @ torch.tensor(s["weights"][1:], dtype=torch.float64).numpy()
    if s["extra"] is not None:
        r = r + s["extra"].cpu().numpy().astype("f8")
    g = r.reshape(case["programs"], case["k"])
    g = g - g[:, :1]   # (the same distances to the mean, and none where all are equal)
    a = (g - g.mean(1)[:, None]) / (g.std(1)[:, None] + s["eps"])
    return {"reward": r, "advantage": a.reshape(-1)}


def exact(case, seed):
    return {"policy": _exact_policy, "advantage": _exact_advantage}.get(case["op"], _exact_rows)(case, seed)
