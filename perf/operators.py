"""Performance cases of the language-model operators: what scores or produces a transcript next to the encoders.

  kind "linear"    a linear layer in 8-bit integers with a scale per token and per output channel: from codes that the
                   program already has (qasr_linear_int8), or from floats, quantised token by token in the same call
                   (qasr_linear_int8_dynamic)
  kind "experts"   the same products grouped by expert: rows sorted by expert, ragged groups, some of them empty, each row
                   reading the codes of its token through an index (qasr_experts_int8)
  kind "logprobs"  log probabilities of given tokens, the entropy of the distribution and its top alternatives
                   (qasr_token_logprobs)

Weights are codes of bell-shaped channels with a scale each, activations bell-shaped with a few channels that stand
out, logits bell-shaped with some tokens ahead; all drawn on the GPU from the seed.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "f16": 2, "bf16": 2, "codes": 1}


def listed():
    return [
        # One token through a small layer: the smallest product, latency alone.
        {"name": "linear_token", "kind": "linear", "M": 1, "N": 2048, "K": 2048, "x": "bf16", "y": "bf16", "bias": False},
        # A decoding batch of 32 sequences, one token each: the weights are read once, little else.
        {"name": "linear_decode_b32", "kind": "linear", "M": 32, "N": 11008, "K": 4096, "x": "f16", "y": "f16", "bias": False},
        # Feed-forward layer of the Conformer-shaped configuration, 16 utterances of 400 frames, codes in hand.
        {"name": "linear_conformer", "kind": "linear", "M": 6400, "N": 2048, "K": 512, "x": "codes", "y": "f32", "bias": True},
        # A prompt of odd length through a layer whose sizes are multiples of nothing.
        {"name": "linear_odd", "kind": "linear", "M": 777, "N": 1029, "K": 1003, "x": "f32", "y": "f32", "bias": True},
        # Prompts of 8192 tokens through a wide layer: the largest product.
        {"name": "linear_prompt", "kind": "linear", "M": 8192, "N": 14336, "K": 4096, "x": "codes", "y": "bf16", "bias": False},
        # Four sequences decode one token each, four experts of 32 per token.
        {"name": "experts_decode", "kind": "experts", "T": 4, "A": 4, "E": 32, "N": 2048, "K": 1024, "tail": 0, "y": "bf16",
         "bias": False},
        # A prompt of 2048 tokens, eight experts of 64 per token.
        {"name": "experts_prompt", "kind": "experts", "T": 2048, "A": 8, "E": 64, "N": 2816, "K": 2048, "tail": 0, "y": "bf16",
         "bias": False},
        # Odd sizes, rows behind the last group that stay as they were.
        {"name": "experts_odd", "kind": "experts", "T": 501, "A": 2, "E": 7, "N": 1001, "K": 520, "tail": 5, "y": "f32",
         "bias": True},
        # Confidence of every frame of 32 utterances over the 29 classes of the encoders' last layer.
        {"name": "logprobs_frames", "kind": "logprobs", "rows": 25600, "V": 29, "x": "f32", "n": 1, "top": 3, "masked": 0.0},
        # One decoded token over a large vocabulary with its twenty best alternatives.
        {"name": "logprobs_token", "kind": "logprobs", "rows": 1, "V": 128256, "x": "f32", "n": 1, "top": 20, "masked": 0.0},
        # A decoding batch under a constraint: nine tenths of the vocabulary are masked.
        {"name": "logprobs_masked_b64", "kind": "logprobs", "rows": 64, "V": 151936, "x": "f16", "n": 1, "top": 20, "masked": 0.9},
        # Scoring hypotheses of 4096 tokens over a vocabulary of odd size, five alternatives.
        {"name": "logprobs_prompt", "kind": "logprobs", "rows": 4096, "V": 50257, "x": "bf16", "n": 2, "top": 5, "masked": 0.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A layer's width: a multiple of 64 mostly, else as it falls."""
    w = _log_int(rng, lo, hi)
    return w if rng.random() < 0.3 else max(64, w // 64 * 64)


def draw(rng):
    kind = rng.choices(["linear", "experts", "logprobs"], [5, 3, 4])[0]
    if kind == "linear":
        N, K = _width(rng, 64, 14336), _width(rng, 64, 8192)
        M = _log_int(rng, 1, min(8192, (1 << 38) // (N * K)))
        return {"kind": kind, "M": M, "N": N, "K": K, "x": rng.choice(["codes", "f32", "f16", "bf16"]),
                "y": rng.choice(["f32", "f16", "bf16"]), "bias": rng.random() < 0.5}
    if kind == "experts":
        E = _log_int(rng, 2, 128)
        A = rng.choice([1, 2, 4, 8])
        N, K = _width(rng, 64, 4096), _width(rng, 64, 4096)
        while E * N * K > 300 << 20:
            N, K = max(64, N // 2), max(64, K // 2)
        return {"kind": kind, "T": _log_int(rng, 1, 2048), "A": min(A, E), "E": E, "N": N, "K": K,
                "tail": rng.choice([0, 0, 3]), "y": rng.choice(["f32", "f16", "bf16"]), "bias": rng.random() < 0.3}
    V = _log_int(rng, 16, 200000)
    x = rng.choice(["f32", "f16", "bf16"])
    return {"kind": kind, "rows": _log_int(rng, 1, min(32768, (100 << 20) // V)), "V": V, "x": x, "n": rng.choice([0, 1, 1, 4]),
            "top": min(V, rng.choice([0, 1, 5, 20, 64])), "masked": rng.choice([0.0, 0.0, 0.5, 0.99])}


# ---- inputs

class _Random:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + 17)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device="cuda")

    def integers(self, lo, hi, *shape):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda", dtype=torch.int32)

    def codes(self, *shape):
        return self.normal(*shape).mul_(36).round_().clamp_(-127, 127).to(torch.int8)

    def scales(self, *shape):
        return self.uniform(*shape).mul_(0.01).add_(0.002)


def _popularity(E):
    """How often each expert is chosen: some several times as often as others."""
    p = [1.0 / (3 + (7 * e) % E) ** 0.5 for e in range(E)]
    return [v / sum(p) for v in p]


def _prepare_linear(c, r):
    M, N, K = c["M"], c["N"], c["K"]
    st = {"w": r.codes(N, K), "w_scale": r.scales(N), "bias": r.normal(N) if c["bias"] else None,
          "y": torch.empty(M, N, dtype=_TYPES[c["y"]], device="cuda")}
    if c["x"] == "codes":
        st["x"], st["x_scale"] = r.codes(M, K), r.scales(M)
    else:
        x = r.normal(M, K) * r.normal(M, 1).abs().add_(0.5)
        x[:, r.integers(0, K, max(1, K // 256)).long()] *= 8
        st["x"] = x.to(_TYPES[c["x"]])
    if own:
        import paper_2103_16827_amd as Q
        st["workspace"] = torch.empty(Q.linear_workspace_bytes(M, K), dtype=torch.int8, device="cuda")
    return st


def _prepare_experts(c, r):
    T, A, E, N, K = c["T"], c["A"], c["E"], c["N"], c["K"]
    # each token's A experts: the largest of log p + Gumbel noise
    noise = -(-r.uniform(T, E).clamp_(1e-9, 1 - 1e-7).log()).log()
    chosen = (noise + torch.tensor(_popularity(E), device="cuda").log()).topk(A, dim=1).indices.reshape(-1)
    order = chosen.sort(stable=True).indices
    sizes = torch.bincount(chosen, minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = sizes.cumsum(0)
    return {"x": r.codes(T, K), "x_scale": r.scales(T), "w": r.codes(E, N, K), "w_scale": r.scales(E, N),
            "bias": r.normal(E, N) if c["bias"] else None, "offsets": offsets, "index": (order // A).to(torch.int32),
            "expert": chosen[order], "most": int(sizes.max()),
            "y": torch.ones(T * A + c["tail"], N, dtype=_TYPES[c["y"]], device="cuda")}


def _prepare_logprobs(c, r):
    rows, V = c["rows"], c["V"]
    x = r.normal(rows, V).mul_(2.5)
    ahead = r.integers(0, V, rows, 8).long()
    x.scatter_add_(1, ahead, r.uniform(rows, 8).mul_(9))
    tokens = ahead[:, :4].clone()
    if c["masked"]:
        x.masked_fill_(r.uniform(1, V).lt(c["masked"]), float("-inf"))   # the same constraint for every row
        x[:, 0] = 0.0                                                    # (the end of the text stays allowed)
    tokens[: rows // 8, 0] = r.integers(0, V, rows // 8).long()
    st = {"x": x.to(_TYPES[c["x"]]), "tokens": tokens[:, : c["n"]].to(torch.int32).contiguous(), "top": c["top"],
          "logprob": torch.empty(rows, c["n"], device="cuda"), "entropy": torch.empty(rows, device="cuda"),
          "top_ids": torch.empty(rows, c["top"], dtype=torch.int32, device="cuda"),
          "top_logprob": torch.empty(rows, c["top"], device="cuda")}
    if own:
        import paper_2103_16827_amd as Q
        st["workspace"] = torch.empty(Q.logprobs_workspace_bytes(rows, V, c["top"]), dtype=torch.int8, device="cuda")
    return st


def prepare(case, seed):
    r = _Random(seed)
    st = {"linear": _prepare_linear, "experts": _prepare_experts, "logprobs": _prepare_logprobs}[case["kind"]](case, r)
    st["kind"] = case["kind"]
    return st


# ---- the plain forms

def _quantize_plain(x):
    """Codes (as floats) and scales of each row: S = max|x| / 127, codes round(x / S)."""
    x = x.float()
    a = x.abs().amax(1, keepdim=True)
    S = torch.where(a > 0, (a / 127).clamp_min(2.0 ** -126), torch.ones_like(a))
    return (x / S).clamp(-127, 127).round(), S


def _linear_plain(st):
    if "x_scale" in st:
        q, S = st["x"].float(), st["x_scale"][:, None]
    else:
        q, S = _quantize_plain(st["x"])
    y = (q @ st["w"].float().t()) * S * st["w_scale"]
    if st["bias"] is not None:
        y = y + st["bias"]
    return y.to(st["y"].dtype)


def _experts_plain(st):
    """Groups padded to the largest one, one batched product, and the rows back in their order."""
    expert, index, y = st["expert"], st["index"].long(), st["y"]
    rows, E, most = index.numel(), st["w"].shape[0], st["most"]
    place = torch.arange(rows, device="cuda") - st["offsets"].long()[expert]
    q = torch.zeros(E, most, st["x"].shape[1], device="cuda")
    q[expert, place] = st["x"][index].float()
    v = torch.bmm(q, st["w"].float().transpose(1, 2).contiguous())[expert, place]
    v = v * st["x_scale"][index][:, None] * st["w_scale"][expert]
    if st["bias"] is not None:
        v = v + st["bias"][expert]
    y[:rows] = v.to(y.dtype)
    return y


def _logprobs_plain(st):
    x = st["x"].float()
    d = x - x.amax(1, keepdim=True)
    e = d.exp()
    s = e.sum(1, keepdim=True)
    entropy = s.log() - torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1, keepdim=True) / s
    lp = d - s.log()
    out = {"logprob": lp.gather(1, st["tokens"].long()), "entropy": entropy[:, 0]}
    if st["top"]:
        # one 64-bit key for each logit: its order above, the lower index first below
        bits = (x + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = order * (1 << 32) + (x.shape[1] - 1 - torch.arange(x.shape[1], device="cuda"))
        ids = key.topk(st["top"], dim=1).indices
        out["top_ids"], out["top_logprob"] = ids.to(torch.int32), lp.gather(1, ids)
    return out


def run(state):
    kind = state["kind"]
    if own:
        import paper_2103_16827_amd as Q
        if kind == "linear":
            if "x_scale" in state:
                return Q.linear_int8(state["x"], state["x_scale"], state["w"], state["w_scale"], state["bias"], state["y"])
            return Q.linear_int8_dynamic(state["x"], state["w"], state["w_scale"], state["bias"], state["y"], state["workspace"])
        if kind == "experts":
            return Q.experts_int8(state["x"], state["x_scale"], state["offsets"], state["index"], state["w"], state["w_scale"],
                                  state["bias"], state["y"])
        Q.token_logprobs(state["x"], state["tokens"], state["logprob"], state["entropy"], state["top_ids"],
                         state["top_logprob"], state["workspace"])
        out = {"logprob": state["logprob"], "entropy": state["entropy"]}
        if state["top"]:
            out["top_ids"], out["top_logprob"] = state["top_ids"], state["top_logprob"]
        return out
    return {"linear": _linear_plain, "experts": _experts_plain, "logprobs": _logprobs_plain}[kind](state)


# ---- what a pass cannot do without

def work(case):
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        scales = 4 * N * (2 if case["bias"] else 1) + (4 * M if case["x"] == "codes" else 0)
        return {"bytes": M * K * _SIZE[case["x"]] + N * K + scales + M * N * _SIZE[case["y"]], "flops": 2 * M * N * K}
    if case["kind"] == "experts":
        rows, N, K = case["T"] * case["A"], case["N"], case["K"]
        # experts that have rows, on average
        busy = sum(1 - (1 - p) ** rows for p in _popularity(case["E"]))
        per = N * K + 4 * N * (2 if case["bias"] else 1)
        return {"bytes": int(case["T"] * (K + 4) + 4 * (rows + case["E"] + 1) + busy * per + rows * N * _SIZE[case["y"]]),
                "flops": 2 * rows * N * K}
    rows, V = case["rows"], case["V"]
    # per logit: a difference, an exponential, two sums and a comparison
    return {"bytes": rows * (V * _SIZE[case["x"]] + 8 * case["n"] + 4 + 8 * case["top"]), "flops": 6 * rows * V}


# ---- the operators' definitions in 64 bits

def _codes_exact(x):
    """Scales are single-precision numbers, and so is the quotient that is rounded: the code is defined by them."""
    x = x.double()
    a = x.abs().max(1).values
    S = torch.where(a > 0, (a / 127).float().double().clamp(min=2.0 ** -126), torch.ones_like(a))
    q = torch.round((x / S[:, None]).float().double())
    return torch.clamp(q, -127, 127), S


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "linear":
        if case["x"] == "codes":
            q, S = st["x"].double(), st["x_scale"].double()
        else:
            q, S = _codes_exact(st["x"])
        acc = torch.matmul(q, st["w"].double().t())
        y = acc * torch.outer(S, st["w_scale"].double())
        return y if st["bias"] is None else y + st["bias"].double()
    if case["kind"] == "experts":
        y = st["y"].double()
        ends = st["offsets"].tolist()
        for e in range(case["E"]):
            lo, hi = ends[e], ends[e + 1]
            if hi > lo:
                tok = st["index"][lo:hi].long()
                left = st["x"][tok].double() * st["x_scale"][tok].double()[:, None]
                right = st["w"][e].double() * st["w_scale"][e].double()[:, None]
                y[lo:hi] = torch.matmul(left, right.t())
                if st["bias"] is not None:
                    y[lo:hi] += st["bias"][e].double()
        return y
    x = st["x"].double()
    lp = torch.log_softmax(x, 1)
    p = lp.exp()
    out = {"logprob": torch.gather(lp, 1, st["tokens"].long()), "entropy": -torch.special.xlogy(p, p).sum(1)}
    if case["top"]:
        ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, : case["top"]]
        out["top_ids"], out["top_logprob"] = ids.to(torch.int32), torch.gather(lp, 1, ids)
    return out
