"""A prompt's attention, the weight it leaves on its positions, and the log probabilities of
tokens, as cases that can be timed.

A case is a dict of plain values.  Three kinds of work:

  attend    causal attention of packed prompts: sequences of different lengths one after the
            other in the rows of a fused projection's output, grouped heads.
  weigh     the attention weight that every position of those prompts received from the last
            `last` rows of its sequence, for every key/value head: what a cache's rows start with.
  logprobs  rows of logits: the log probabilities of given tokens, the entropy, the most likely
            tokens (ties to the lowest) and their log probabilities.

Inputs are seeded: keys have an offset for each channel and rows of unequal size, queries lean
towards the offsets; logits have a frequency for each token and rows of unequal sharpness.
Lengths and row counts follow from the case alone, so that its work does.
"""
import math

import torch

own = False

RAW = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # one short prompt of a small model: a launch's latency
        dict(name="prompt_short", kind="attend", B=1, n=133, ragged=False, Hq=8, H=2, D=64),
        # requests with their tool lists, admitted together, 375 to 1,500 tokens each
        dict(name="prompts_batch", kind="attend", B=48, n=1500, ragged=True, Hq=32, H=8, D=128),
        # one conversation's history, an odd length
        dict(name="prompt_8k", kind="attend", B=1, n=8191, ragged=False, Hq=32, H=8, D=128),
        # one document
        dict(name="prompt_16k", kind="attend", B=1, n=16384, ragged=False, Hq=32, H=8, D=128),
        # a very long document over the few heads that a shard of a model holds
        dict(name="prompt_64k", kind="attend", B=1, n=65533, ragged=False, Hq=2, H=1, D=128),
        # what a short prompt's rows start with
        dict(name="weigh_short", kind="weigh", B=1, n=133, ragged=False, Hq=8, H=2, D=64, last=133),
        # four conversations judged by their last 64 rows
        dict(name="weigh_recent", kind="weigh", B=4, n=8191, ragged=True, Hq=32, H=8, D=128, last=64),
        # a conversation judged by every row
        dict(name="weigh_all", kind="weigh", B=1, n=8192, ragged=False, Hq=32, H=8, D=128, last=8192),
        # a token of one request, a float32 head
        dict(name="token_one", kind="logprobs", B=1, N=1, V=32003, raw="f32", M=1, top=8, ragged=False),
        # one verified tree of 60 nodes and the root: predictions and the drafts' log probabilities
        dict(name="tree_one", kind="logprobs", B=1, N=61, V=131072, raw="bf16", M=1, top=1, ragged=False),
        # 32 trees of up to 61 nodes, eight alternatives kept of each node
        dict(name="tree_batch", kind="logprobs", B=32, N=61, V=131072, raw="bf16", M=1, top=8, ragged=True),
        # four prompts' own tokens scored, an odd vocabulary
        dict(name="score_prompts", kind="logprobs", B=4, N=1021, V=50021, raw="f32", M=1, top=0, ragged=True),
    ]


SCORES = 32 * 16384 * 16384  # of the largest listed case
LOGITS = 32 * 61 * 131072


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "weigh", "logprobs", "logprobs"])
    if kind == "logprobs":
        raw = rng.choice(["bf16", "bf16", "f32"])
        V = _log(rng, 300, 262144)
        B = rng.choice([1, 1, 2, 5, 8, 32])
        most = LOGITS // (B * V * (2 if raw == "f32" else 1))
        return dict(kind=kind, B=B, N=_log(rng, 1, max(1, min(1024, most))), V=V, raw=raw,
                    M=rng.choice([0, 1, 1, 1, 4]), top=rng.choice([0, 1, 1, 5, 8, 20, 64]),
                    ragged=B > 1 and rng.random() < 0.7)
    D = rng.choice([64, 128, 128, 128, rng.choice([80, 96, 40])])
    H = rng.choice([1, 2, 4, 8, 8, 12])
    Hq = H * rng.choice([1, 2, 4, 4, 5, 7, 8])
    B = rng.choice([1, 1, 2, 3, 8, 17, 48])
    n = _log(rng, 1, min(65536, math.isqrt(SCORES // (B * Hq))))
    case = dict(kind=kind, B=B, n=n, ragged=B > 1 and rng.random() < 0.8, Hq=Hq, H=H, D=D)
    if kind == "weigh":
        case["last"] = rng.choice([1, 16, 64, 64, 256, n])
    return case


def _lens(case):
    n = case["n"]
    return [n - (b * 7919) % (3 * n // 4 + 1) if case["ragged"] else n for b in range(case["B"])]


def _counts(case):
    """Rows of logits of each request."""
    N = case["N"]
    return [N - (b * 5) % (N // 3 + 1) if case["ragged"] else N for b in range(case["B"])]


def work(case):
    """Bytes and operations of one pass: inputs read once, outputs written once."""
    if case["kind"] == "logprobs":
        rows, e = sum(_counts(case)), 4 if case["raw"] == "f32" else 2
        out = case["B"] * case["N"] * (8 * case["M"] + 4 + 8 * case["top"])
        return {"bytes": rows * case["V"] * e + out, "flops": 5 * rows * case["V"]}
    Hq, H, D, lens = case["Hq"], case["H"], case["D"], _lens(case)
    if case["kind"] == "attend":
        return {"bytes": sum(lens) * (4 * Hq * D + 4 * H * D + 4 * Hq),
                "flops": 4 * D * Hq * sum(n * (n + 1) // 2 for n in lens)}
    seen = [min(case["last"], n) for n in lens]
    return {"bytes": sum(lens) * H * (2 * D + 4) + sum(seen) * Hq * (2 * D + 4),
            "flops": 2 * D * Hq * sum(r * n - r * (r - 1) // 2 for r, n in zip(seen, lens))}


# ------------------------------------------------------------------ inputs
def _dev():
    return torch.device("cuda")


def _gen(seed, part):
    g = torch.Generator(device=_dev())
    g.manual_seed((seed * 1000003 + part) & 0x7FFFFFFFFFFF)
    return g


def _normal(seed, part, *shape):
    return torch.randn(shape, generator=_gen(seed, part), device=_dev())


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device=_dev())


def _starts(case):
    at = [0]
    for n in _lens(case):
        at.append(at[-1] + n)
    return at


def _rows(case, seed):
    """q, k, v (T, heads, D): views of one projection's output."""
    T, Hq, H, D = _starts(case)[-1], case["Hq"], case["H"], case["D"]
    offset = 1.5 * _normal(seed, 1, H, D)
    size = torch.exp(0.3 * _normal(seed, 2, T, H, 1))
    x = torch.empty((T, Hq + 2 * H, D), dtype=torch.bfloat16, device=_dev())
    q, k, v = x.split([Hq, H, H], dim=1)
    lean = 0.2 * offset.repeat_interleave(Hq // H, 0)
    q.copy_(1.3 * _normal(seed, 3, T, Hq, D) + lean)
    k.copy_(_normal(seed, 4, T, H, D) * size + offset)
    v.copy_(_normal(seed, 5, T, H, D) * size)
    return q, k, v


def _logits(case, seed):
    """Logits (B, N, V), given tokens (B, N, M)."""
    B, N, V = case["B"], case["N"], case["V"]
    x = _normal(seed, 6, B, N, V).add_(1.5 * _normal(seed, 7, V)).mul_(torch.exp(0.5 * _normal(seed, 8, B, N, 1)))
    given = torch.randint(V, (B, N, case["M"]), generator=_gen(seed, 9), device=_dev())
    if case["M"]:  # the first is what the model expects, by a margin that differs
        x.scatter_add_(2, given[:, :, :1], 4 + 4 * _normal(seed, 10, B, N, 1))
    return x.to(RAW[case["raw"]]), given.to(torch.int32)


def prepare(case, seed):
    st = dict(kind=case["kind"], case=case)
    if case["kind"] == "logprobs":
        st["logits"], st["tokens"] = _logits(case, seed)
        st["counts"] = _int(_counts(case))
        return st
    st["q"], st["k"], st["v"] = _rows(case, seed)
    st["starts"] = _int(_starts(case))
    st["scale"] = 1.0 / math.sqrt(case["D"])
    if case["kind"] == "weigh":
        st["lse"] = _lse_of(st)
    return st


def _lse_of(st):
    """What the forward gave with the queries."""
    case = st["case"]
    s, at, live = _scores(st, case["n"])
    s = s.logsumexp(-1)
    return _packed(s.flatten(1, 2).transpose(1, 2), live)


# ------------------------------------------------------------------ the plain forms
def _padded(st, n):
    """Row numbers (B, n) of every sequence's positions 0 .. n - 1, and which of them it has."""
    first, end = st["starts"][:-1, None].long(), st["starts"][1:, None].long()
    at = first + torch.arange(n, device=first.device)
    return torch.minimum(at, end - 1), at < end


def _packed(x, live):
    """(B, n, ...) -> the rows that are live, one after the other."""
    return x[live]


def _heads(x, at):
    """Rows (T, heads, D) at (B, n) -> (B, heads, n, D) in f32."""
    return x[at].float().transpose(1, 2).contiguous()


def _scores(st, last):
    """Scores (B, H, G, R, n) in f32 of each sequence's last R = min(last, n) rows (aligned at n, the longest's
    length), -inf where a row does not see a key; the rows' numbers (B, R) and which exist."""
    case = st["case"]
    B, H, G, D, n = case["B"], case["H"], case["Hq"] // case["H"], case["D"], case["n"]
    R = min(last, n)
    keys, _ = _padded(st, n)
    first, end = st["starts"][:-1, None].long(), st["starts"][1:, None].long()
    back = torch.arange(R, device=first.device)
    own_rows = torch.clamp(end - first - R, min=0) + back  # position in the sequence
    live = own_rows < end - first
    rows = torch.minimum(first + own_rows, end - 1)
    q = _heads(st["q"], rows).view(B, H, G * R, D)
    k = _heads(st["k"], keys).transpose(2, 3).contiguous()
    s = torch.matmul(q, k).view(B, H, G, R, n)
    s *= st["scale"]
    unseen = torch.arange(n, device=first.device) > own_rows[:, :, None]
    return s.masked_fill_(unseen[:, None, None], -math.inf), rows, live


def _run_plain(st):
    case = st["case"]
    if st["kind"] == "logprobs":
        return _plain_logprobs(st)
    B, H, G, D, n = case["B"], case["H"], case["Hq"] // case["H"], case["D"], case["n"]
    if st["kind"] == "attend":
        s, _, live = _scores(st, n)
        top = s.amax(-1, keepdim=True)
        p = s.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        keys, _ = _padded(st, n)
        o = torch.matmul(p.view(B, H, G * n, n), _heads(st["v"], keys)).view(B, H, G, n, D) / total
        lse = (top + torch.log(total))[..., 0]
        out = o.flatten(1, 2).transpose(1, 2).to(torch.bfloat16)
        return {"out": _packed(out, live), "lse": _packed(lse.flatten(1, 2).transpose(1, 2), live)}
    s, rows, live = _scores(st, case["last"])
    lse = st["lse"][rows].view(B, -1, H, G).permute(0, 2, 3, 1)
    p = s.sub_(lse[..., None]).exp_()
    p *= live[:, None, None, :, None]
    weight = p.sum((2, 3))  # (B, H, n)
    _, held = _padded(st, n)
    return {"weight": _packed(weight.transpose(1, 2), held).T.contiguous()}


def _plain_logprobs(st):
    x, tokens = st["logits"], st["tokens"]
    V, top = st["case"]["V"], st["case"]["top"]
    live = (torch.arange(x.shape[1], device=x.device) < st["counts"][:, None])[..., None]
    none = torch.full((), -math.inf, device=x.device)
    d = x.float()
    m = d.amax(-1, keepdim=True)
    d = d - m
    p = d.exp()
    total = p.sum(-1, keepdim=True)
    log_total = total.log()
    entropy = log_total - (p * d).sum(-1, keepdim=True) / total
    given = torch.gather(d, 2, tokens.long()) - log_total
    # the order (logit descending, token ascending) as one whole number
    bits = (x.float() + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    order = (order << 32) | (V - 1 - torch.arange(V, device=x.device))
    best = torch.topk(order, top, dim=-1).values
    ids = V - 1 - (best & 0xFFFFFFFF)
    alternatives = torch.gather(d, 2, ids) - log_total
    return {"logprob": torch.where(live, given, none), "entropy": torch.where(live, entropy, 0.0)[..., 0],
            "top_tokens": torch.where(live, ids, -1).to(torch.int32),
            "top_logprobs": torch.where(live, alternatives, none)}


# ------------------------------------------------------------------ a pass
def run(st):
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    import paper_2608_03839_amd as oil

    case = st["case"]
    if st["kind"] == "attend":
        out, lse = oil.prompt_attend(st["q"], st["k"], st["v"], st["starts"], scale=st["scale"])
        return {"out": out, "lse": lse}
    if st["kind"] == "weigh":
        return {"weight": oil.prompt_weigh(st["q"], st["k"], st["lse"], st["starts"], last=case["last"],
                                           scale=st["scale"])}
    logprob, entropy, tokens, logprobs = oil.token_logprobs(st["logits"], st["tokens"], top=case["top"],
                                                            n_rows=st["counts"])
    return {"logprob": logprob, "entropy": entropy, "top_tokens": tokens, "top_logprobs": logprobs}


# ------------------------------------------------------------------ in 64 bits, from the definition
def _exact_prompts(case, seed):
    """Attention (T, Hq, D) and lse (T, Hq) of every sequence, a head and a block of rows at a time."""
    q, k, v = (x.double() for x in _rows(case, seed))
    T, Hq, D = q.shape
    out, lse = torch.empty_like(q), torch.empty((T, Hq), dtype=torch.float64, device=q.device)
    block = 4096
    for a, z in zip(_starts(case), _starts(case)[1:]):
        for head in range(Hq):
            h = head // (Hq // case["H"])
            for i in range(a, z, block):
                j = min(z, i + block)
                s = q[i:j, head] @ k[a:j, h].T / math.sqrt(D)
                s[:, i - a:] += torch.full((j - i, j - i), -math.inf, dtype=torch.float64, device=q.device).triu(1)
                lse[i:j, head] = torch.logsumexp(s, 1)
                out[i:j, head] = torch.softmax(s, 1) @ v[a:j, h]
    return {"out": out, "lse": lse}


def _exact_weight(case, seed):
    st = prepare(case, seed)
    q, k, lse = st["q"].double(), st["k"].double(), st["lse"].double()
    T, Hq, D = q.shape
    weight = torch.zeros((case["H"], T), dtype=torch.float64, device=q.device)
    for a, z in zip(_starts(case), _starts(case)[1:]):
        first = max(a, z - case["last"])
        for head in range(Hq):
            for i in range(first, z, 4096):
                j = min(z, i + 4096)
                p = torch.exp(q[i:j, head] @ k[a:j, head // (Hq // case["H"])].T / math.sqrt(D) - lse[i:j, head, None])
                p[:, i - a:] = p[:, i - a:].tril()
                weight[head // (Hq // case["H"]), a:j] += p.sum(0)
    return {"weight": weight}


def _exact_logprobs(case, seed):
    x, tokens = _logits(case, seed)
    B, N, M, k = case["B"], case["N"], case["M"], case["top"]
    full = dict(dtype=torch.float64, device=x.device)
    got = {"logprob": torch.full((B, N, M), -math.inf, **full), "entropy": torch.zeros((B, N), **full),
           "top_tokens": torch.full((B, N, k), -1, dtype=torch.int64, device=x.device),
           "top_logprobs": torch.full((B, N, k), -math.inf, **full)}
    for b, m in enumerate(_counts(case)):
        for i in range(0, m, 64):
            at = slice(i, min(m, i + 64))
            y = torch.log_softmax(x[b, at].double(), -1)
            got["logprob"][b, at] = y.gather(1, tokens[b, at].long())
            got["entropy"][b, at] = -(y.exp() * y).sum(1)
            if k:
                order = torch.sort(x[b, at].double(), dim=1, descending=True, stable=True).indices[:, :k]
                got["top_tokens"][b, at] = order
                got["top_logprobs"][b, at] = y.gather(1, order)
    return got


def exact(case, seed):
    if case["kind"] == "logprobs":
        return _exact_logprobs(case, seed)
    if sum(n * n for n in _lens(case)) * case["Hq"] > SCORES:
        return None
    return _exact_prompts(case, seed) if case["kind"] == "attend" else _exact_weight(case, seed)
