"""The operators that a server of many requests runs in a decode step beside those of perf/operators.py, each in its plain form and
as the framework's call:

  shared    decode attention over the paged 4-bit cache for a batch whose sequences share long prefixes in groups: a prefix is read
            once for its group
  adapters  low-rank adapters of many requests at once, added to the output of a projection that they share
  logprobs  log probabilities and ranks of given tokens, the entropy of each row and its most likely tokens

Heads and layers are those of the models that the benchmark measures, and generic ones.
"""
import math

import torch

own = False

D = 128                     # head dimension
PAGE = 64                   # tokens of a page


# ------------------------------------------------------------------------------------------------------------------
# The cases
# ------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # four answers sampled for one prompt, just begun: latency
        dict(name="shared-4x1000+30-h32-8", kind="shared", H=32, Hkv=8, groups=1, members=4, alone=0, prefix=1000, tokens=30),
        # a full batch behind one system prompt, some way into the answers
        dict(name="shared-64x4096+300-h32-8", kind="shared", H=32, Hkv=8, groups=1, members=64, alone=0, prefix=4096, tokens=300),
        # three prompts of a multi-head model, their ends inside pages, beside requests that share nothing
        dict(name="shared-3x11+4x777+150-h32-32", kind="shared", H=32, Hkv=32, groups=3, members=11, alone=4, prefix=777, tokens=150),
        # many questions about one long document on the largest model: the most work in one pass
        dict(name="shared-200x16000+100-h64-8", kind="shared", H=64, Hkv=8, groups=1, members=200, alone=0, prefix=16000, tokens=100),
        # generation for one user: launches and latency only
        dict(name="adapters-1-n4096-k4096-r16", kind="adapters", M=1, N=4096, K=4096, rank=16, adapters=8, used=1, prompts=False),
        # a full batch on the fused QKV projection of a grouped-query model, rows of many adapters and of none in any order
        dict(name="adapters-64-n6144-k4096-r16", kind="adapters", M=64, N=6144, K=4096, rank=16, adapters=40, used=23, prompts=False),
        # ragged prompts of five requests, a rank that fills no tile
        dict(name="adapters-1733-n11008-k4096-r8", kind="adapters", M=1733, N=11008, K=4096, rank=8, adapters=8, used=5, prompts=True),
        # prompts on the widest layer, large adapters: the most work in one pass
        dict(name="adapters-4096-n28672-k8192-r64", kind="adapters", M=4096, N=28672, K=8192, rank=64, adapters=6, used=3, prompts=True),
        # one token of one request
        dict(name="logprobs-1x32000-top5", kind="logprobs", M=1, V=32000, top=5, wide=False, masked=False),
        # a full batch over a large vocabulary, every alternative that an interface offers
        dict(name="logprobs-64x128256-top20", kind="logprobs", M=64, V=128256, top=20, wide=False, masked=True),
        # logits kept in 32 bits, an odd vocabulary, answers that are only scored
        dict(name="logprobs-37x50257-fp32", kind="logprobs", M=37, V=50257, top=0, wide=True, masked=False),
        # every token of a prompt scored: the most work in one pass
        dict(name="logprobs-4001x32000-top1", kind="logprobs", M=4001, V=32000, top=1, wide=False, masked=False),
    ]


_HEADS = ((32, 32), (32, 8), (64, 8), (28, 4), (40, 8), (16, 1), (9, 3))
_LAYERS = ((4096, 4096), (6144, 4096), (11008, 4096), (4096, 11008), (8192, 8192), (5120, 5120), (1032, 776), (28672, 8192))


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(("shared", "adapters", "logprobs"))
    if kind == "shared":
        H, Hkv = rng.choice(_HEADS)
        groups = rng.choice((1, 1, 2, 5))
        members = _log_int(rng, 2, 200 // groups)
        alone = rng.choice((0, 0, rng.randint(1, 9)))
        prefix = _log_int(rng, 1, max(1, min(16000, 200 * 15000 * 64 // (groups * members * H))))
        tokens = _log_int(rng, 1, min(600, 400000 // ((groups * members + alone) * Hkv)))
        return dict(kind=kind, H=H, Hkv=Hkv, groups=groups, members=members, alone=alone, prefix=prefix, tokens=tokens)
    if kind == "adapters":
        N, K = rng.choice(_LAYERS)
        prompts = rng.random() < 0.5
        M = _log_int(rng, 100, min(4096, 4096 * 36000 // (N + K))) if prompts else _log_int(rng, 1, 256)
        adapters = _log_int(rng, 1, 64)
        return dict(kind=kind, M=M, N=N, K=K, rank=rng.choice((8, 16, 16, 24, 32, 64)), adapters=adapters,
                    used=rng.randint(1, min(adapters, 8 if prompts else M)), prompts=prompts)
    V = _log_int(rng, 1000, 160000)
    wide = rng.random() < 0.3
    return dict(kind=kind, M=_log_int(rng, 1, min(4096, 128000000 // (V * (2 if wide else 1)))), V=V, top=rng.choice((0, 1, 5, 20, 32)),
                wide=wide, masked=rng.random() < 0.3)


def _lengths(B, longest):
    """B lengths from `longest` down to half of it."""
    return [longest - (longest // 2) * b // max(B - 1, 1) for b in range(B)]


def _batch(case):
    """Members of the groups [(first, behind the last, prefix)], and of every sequence what it has of a prefix and in all."""
    n, G = case["members"], case["groups"]
    groups = [(g * n, (g + 1) * n, p) for g, p in enumerate(_lengths(G, case["prefix"]))]
    B = G * n + case["alone"]
    shared = [p for _, _, p in groups for _ in range(n)] + [0] * case["alone"]
    total = [s + t for s, t in zip(shared, _lengths(B, case["tokens"]))]
    if n >= 8:
        total[n - 1] = shared[n - 1] = 0    # a slot of the first group that no request holds
    return groups, shared, total


# ------------------------------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=g.device, dtype=torch.float16)


def _keys(g, *shape):
    """Keys [..., Hkv, D] with two large channels in every KV head."""
    k = _normal(g, *shape)
    cols = torch.rand(shape[-2], D, generator=g, device=g.device).topk(2, dim=1).indices
    gain = torch.ones(shape[-2], D, device=g.device, dtype=torch.float16).scatter_(1, cols, 8.0)
    return k * gain


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cumulative(lengths):
    total, out = 0, [0]
    for n in lengths:
        total += n
        out.append(total)
    return out


def _shared_inputs(s, g):
    """Keys and values of each prefix once, then of what every sequence has of its own.  The whole pages of a prefix are the same
    ones in the block tables of its group; its tokens behind them stand in the first member's next page only."""
    groups, shared, total = _batch(s)
    B, Hkv = len(total), s["Hkv"]
    tokens = [t - p for t, p in zip(total, shared)]
    width = max(1, max(-(-max(t, p) // PAGE) for t, p in zip(total, [p for _, _, p in groups] + total)))
    table = torch.full((B, width), -1, dtype=torch.int32)
    need = [p // PAGE for _, _, p in groups] + [-(-t // PAGE) - p // PAGE for t, p in zip(total, shared)]
    s["pages"] = sum(need) + 3
    perm, at = torch.randperm(s["pages"], generator=g, device="cuda").to(torch.int32).cpu(), _cumulative(need)
    for i, (a, e, p) in enumerate(groups):
        for b in range(a, e):
            if shared[b] or b == a:
                table[b, :p // PAGE] = perm[at[i]:at[i] + p // PAGE]
    for b in range(B):
        first, n = shared[b] // PAGE, need[len(groups) + b]
        table[b, first:first + n] = perm[at[len(groups) + b]:at[len(groups) + b] + n]
    s["rows_cu"] = _ints(_cumulative([p for _, _, p in groups] + tokens))
    s["rows_at"] = _ints([0] * len(groups) + shared)
    who = [a for a, _, _ in groups] + list(range(B))
    s["table"] = table.cuda()
    s["rows_table"] = s["table"][torch.tensor(who, device="cuda")].contiguous()
    M = sum(p for _, _, p in groups) + sum(tokens)
    s["k"], s["v"] = _keys(g, M, Hkv, D), _normal(g, M, Hkv, D)
    s["lens"] = _ints(total)
    s["group_cu"] = _ints([a for a, _, _ in groups] + [groups[-1][1]])
    s["prefix_lens"] = _ints([p for _, _, p in groups])
    s["q"] = _normal(g, B, s["H"], D)


def _row_adapters(case, g):
    """The adapter of every row, -1 for none: requests in any order, or whole prompts one behind the other."""
    M, used = case["M"], case["used"]
    names = torch.randperm(case["adapters"], generator=g, device="cuda")[:used]
    if case["prompts"]:
        which = torch.tensor([i for i, n in enumerate(_lengths(used, 1000)) for _ in range(n)], device="cuda")
        which = which[torch.arange(M, device="cuda") * which.numel() // M]
        return names[which].to(torch.int32)
    which = torch.randint(0, used, (M,), generator=g, device="cuda")
    row = names[which].to(torch.int32)
    if M >= 8:                              # requests of the model without an adapter
        row[torch.rand(M, generator=g, device="cuda") < 0.1] = -1
    return row


def _case_inputs(case, seed):
    """What the plain form, the framework's calls and the exact form start from."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    if s["kind"] == "shared":
        _shared_inputs(s, g)
    elif s["kind"] == "adapters":
        M, N, K, r, n = s["M"], s["N"], s["K"], s["rank"], s["adapters"]
        x = _normal(g, M, K)
        x[:, torch.randint(0, K, (max(1, K // 100),), generator=g, device="cuda")] *= 20.0
        s["x"], s["base"] = x, _normal(g, M, N)
        s["a"] = _normal(g, n, r, K) * (1.0 / math.sqrt(K))
        s["b"] = _normal(g, n, N, r) * 0.1
        s["scales"] = torch.rand(n, generator=g, device="cuda") + 0.5
        s["row_adapter"] = _row_adapters(case, g)
    else:
        M, V = s["M"], s["V"]
        # likely tokens a few units above the others: some rows are sure of a token, some of none
        x = torch.randn((M, V), generator=g, device="cuda") * 2.0
        some = torch.randint(0, V, (M, 12), generator=g, device="cuda")
        x.scatter_add_(1, some, torch.rand((M, 12), generator=g, device="cuda") * 16.0)
        given = torch.randint(0, V, (M,), generator=g, device="cuda")
        likely = torch.rand(M, generator=g, device="cuda") < 0.7
        given = torch.where(likely, some[:, 0], given)
        if s["masked"]:                     # a grammar allows some of the tokens, the given one among them
            at = x.gather(1, given[:, None])
            x[::3].masked_fill_(torch.rand((V,), generator=g, device="cuda") < 0.7, -math.inf)
            x.scatter_(1, given[:, None], at)
        s["tokens"] = given.to(torch.int32)
        s["logits"] = x if s["wide"] else x.half()
    return s


def prepare(case, seed):
    s = _case_inputs(case, seed)
    if own:
        from paper_2405_04532_amd import api
    if s["kind"] == "shared":
        B, G = s["q"].shape[0], s["prefix_lens"].numel()
        if own:
            s["pool"] = api.kv4_new_pool(s["pages"], s["Hkv"], "cuda")
            api.kv4_paged_append(s["pool"], s["k"], s["v"], s["rows_table"], s["rows_cu"], s["rows_at"])
            need = api.kv4_shared_attention_workspace_bytes(B, s["H"], s["Hkv"], s["table"].shape[1], G)
            s["workspace"] = api.new_workspace(need, "cuda")
            s["out"] = torch.empty((B, s["H"], D), dtype=torch.float16, device="cuda")
        else:
            s["pool"] = _plain_pool(s["pages"], s["Hkv"])
            _plain_write(s["pool"], s["k"], s["v"], s["rows_table"], s["rows_cu"], s["rows_at"])
        del s["k"], s["v"]                  # the cache holds them
    elif s["kind"] == "adapters" and not own:
        s["rows"] = [torch.nonzero(s["row_adapter"] == n).flatten() for n in range(s["adapters"])]
    elif s["kind"] == "adapters":
        s["plan"] = api.lora_plan(s["row_adapter"], s["adapters"])      # one for all layers of a step
        s["workspace"] = api.new_workspace(api.lora_workspace_bytes(s["M"], s["N"], s["K"], s["rank"], s["adapters"]), "cuda")
        s["out"] = torch.empty_like(s["base"])
    elif own:
        s["workspace"] = api.new_workspace(api.token_logprobs_workspace_bytes(s["M"], s["V"], s["top"], s["logits"].dtype), "cuda")
    return s


# ------------------------------------------------------------------------------------------------------------------
# Plain forms
# ------------------------------------------------------------------------------------------------------------------
def _plain_pool(pages, Hkv):
    """For keys and for values: two codes to a byte [pages, Hkv, PAGE, D / 2], scales and zeros [pages, Hkv, PAGE]."""
    half = lambda: (torch.zeros((pages, Hkv, PAGE, D // 2), dtype=torch.uint8, device="cuda"),  # noqa: E731
                    torch.zeros((pages, Hkv, PAGE), dtype=torch.float16, device="cuda"),
                    torch.zeros((pages, Hkv, PAGE), dtype=torch.float16, device="cuda"))
    return half(), half()


def _plain_write(pool, k, v, table, cu, starts):
    row = torch.arange(k.shape[0], device=cu.device)
    seq = torch.searchsorted(cu[1:].long(), row, right=True)
    pos = starts.long()[seq] + row - cu.long()[seq]
    page, off = table[seq, pos // PAGE].long(), pos % PAGE
    for (codes, scale, zero), x in zip(pool, (k, v)):
        # Eq. 1 with four bits; in 64 bits, since codes are decided at half-integers
        x = x.double()
        lo, hi = x.amin(-1).clamp(max=0.0), x.amax(-1).clamp(min=0.0)
        s = ((hi - lo) / 15.0).half()
        s = torch.where(s == 0, torch.ones_like(s), s)
        z = torch.floor(-lo / s.double() + 0.5).clamp(0.0, 15.0)
        c = torch.floor(x / s.double()[..., None] + z[..., None] + 0.5).clamp(0.0, 15.0).to(torch.uint8)
        codes[page, :, off] = c[..., 0::2] | (c[..., 1::2] << 4)
        scale[page, :, off], zero[page, :, off] = s, z.half()


def _plain_values(codes, scale, zero):
    """Eq. 2 in 32 bits: [..., D / 2] bytes -> [..., D]."""
    c = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).float()
    return (c - zero.float()[..., None]) * scale.float()[..., None]


def _plain_pages(pool, page):
    """Keys and values of pages [..., n] as [..., Hkv, n * PAGE, D]."""
    page = page.long().clamp(min=0)
    return [_plain_values(c[page], s[page], z[page]).transpose(-4, -3).flatten(-3, -2) for c, s, z in pool]


def _plain_shared(s):
    """Scores of the own tokens of all sequences, then those of each group's prefix, one softmax over both."""
    H, Hkv, table = s["H"], s["Hkv"], s["table"]
    B, R = s["q"].shape[0], H // Hkv
    groups, shared, total = _batch(s)
    q = s["q"].float().view(B, Hkv, R, D) / math.sqrt(D)
    lens, first = s["lens"].long(), torch.zeros(B, dtype=torch.long, device="cuda")
    for i, (a, e, _) in enumerate(groups):
        first[a:e] = s["prefix_lens"][i]
    reach = max(-(-t // PAGE) - p // PAGE for t, p in zip(total, shared))
    index = first[:, None] // PAGE + torch.arange(reach, device="cuda")
    t = (index[..., None] * PAGE + torch.arange(PAGE, device="cuda")).flatten(1)
    seen = ((t >= first[:, None]) & (t < lens[:, None]))[:, None, None]
    k, v = _plain_pages(s["pool"], table.gather(1, index.clamp(max=table.shape[1] - 1)))
    score = torch.matmul(q, k.transpose(-1, -2).contiguous()).masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    before = []
    for a, e, p in groups:
        pk, pv = _plain_pages(s["pool"], table[a, :-(-p // PAGE)])
        rows = q[a:e].transpose(0, 1).reshape(Hkv, (e - a) * R, D)
        ps = torch.matmul(rows, pk[:, :p].transpose(-1, -2).contiguous()).view(Hkv, e - a, R, p).transpose(0, 1)
        ps = ps.masked_fill((torch.arange(p, device="cuda") >= lens[a:e, None])[:, None, None], -math.inf)
        top[a:e] = torch.maximum(top[a:e], ps.amax(-1, keepdim=True))
        before.append((ps, pv[:, :p]))
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    weight = torch.exp(score - top)
    total_weight, out = weight.sum(-1, keepdim=True), torch.matmul(weight, v)
    for (a, e, p), (ps, pv) in zip(groups, before):
        weight = torch.exp(ps - top[a:e])
        total_weight[a:e] += weight.sum(-1, keepdim=True)
        weight = weight.transpose(0, 1).reshape(Hkv, (e - a) * R, p)
        out[a:e] += torch.matmul(weight, pv).view(Hkv, e - a, R, D).transpose(0, 1)
    return (out / torch.where(total_weight > 0, total_weight, torch.ones_like(total_weight))).view(B, H, D).half()


def _plain_adapters(s):
    """Every adapter's rows in turn, as far as any row has it."""
    out = s["base"].float()
    for n, rows in enumerate(s["rows"]):
        if not rows.numel():
            continue
        low = torch.matmul(s["x"][rows].float(), s["a"][n].float().T)
        out[rows] += s["scales"][n] * torch.matmul(low, s["b"][n].float().T)
    return out.half()


def _plain_logprobs(s):
    x, top = s["logits"].float(), s["top"]
    given = s["tokens"].long()[:, None]
    d = x - x.amax(-1, keepdim=True)
    e = torch.exp(d)
    total = e.sum(-1, keepdim=True)
    log_total = torch.log(total)
    entropy = log_total - torch.where(e > 0, e * d, torch.zeros_like(d)).sum(-1, keepdim=True) / total
    index = torch.arange(x.shape[1], device=x.device)
    at = x.gather(1, given)
    rank = 1 + ((x > at) | ((x == at) & (index < given))).sum(-1)
    out = dict(logprob=(d.gather(1, given) - log_total)[:, 0], rank=rank.to(torch.int32), entropy=entropy[:, 0])
    if top:
        ids = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :top]
        out["top_ids"], out["top_logprobs"] = ids.to(torch.int32), d.gather(1, ids) - log_total
    return out


# ------------------------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------------------------
def run(s):
    kind = s["kind"]
    if own:
        from paper_2405_04532_amd import api
        if kind == "shared":
            return dict(out=api.kv4_shared_attention_decode(s["q"], s["pool"], s["table"], s["lens"], s["group_cu"], s["prefix_lens"],
                                                            s["Hkv"], out=s["out"], workspace=s["workspace"]))
        if kind == "adapters":
            return dict(out=api.lora_add(s["base"], s["x"], s["a"], s["b"], s["plan"], scales=s["scales"], out=s["out"],
                                         workspace=s["workspace"]))
        logprob, rank, entropy, ids, top = api.token_logprobs(s["logits"], s["tokens"], top=s["top"], workspace=s["workspace"])
        out = dict(logprob=logprob, rank=rank, entropy=entropy)
        if s["top"]:
            out["top_ids"], out["top_logprobs"] = ids, top
        return out
    if kind == "logprobs":
        return _plain_logprobs(s)
    return dict(out=_plain_shared(s) if kind == "shared" else _plain_adapters(s))


# ------------------------------------------------------------------------------------------------------------------
# The definitions in 64 bits
# ------------------------------------------------------------------------------------------------------------------
def _exact_cached(x):
    """The numbers that a 4-bit cache holds for the FP16 vectors x[..., D]."""
    x = x.double()
    zero = torch.zeros((), dtype=torch.float64, device=x.device)
    low, high = torch.minimum(x.min(-1, keepdim=True).values, zero), torch.maximum(x.max(-1, keepdim=True).values, zero)
    step = ((high - low) / 15).to(torch.float16).double()
    step[step == 0] = 1.0
    shift = (0.5 - low / step).floor().clip(0, 15)
    return ((x / step + shift + 0.5).floor().clip(0, 15) - shift) * step


def _exact_shared(s):
    """A sequence at a time, over the prefix and its own tokens in one piece."""
    groups, shared, total = _batch(s)
    B, H, Hkv = len(total), s["H"], s["Hkv"]
    k, v, cu = _exact_cached(s["k"]), _exact_cached(s["v"]), s["rows_cu"].tolist()
    out = torch.zeros((B, H, D), dtype=torch.float64, device="cuda")
    for b in range(B):
        if not total[b]:
            continue
        g = next((i for i, (a, e, _) in enumerate(groups) if a <= b < e), None)
        own_rows = slice(cu[len(groups) + b], cu[len(groups) + b + 1])
        parts = [own_rows] if g is None else [slice(cu[g], cu[g + 1]), own_rows]
        kb, vb = (torch.cat([x[p] for p in parts]).permute(1, 2, 0) for x in (k, v))       # [Hkv, D, t]
        a = torch.bmm(s["q"][b].double().view(Hkv, -1, D), kb.contiguous()) * D ** -0.5
        out[b] = torch.bmm(torch.softmax(a, -1), vb.transpose(1, 2).contiguous()).view(H, D)
    return dict(out=out)


def _exact_adapters(s):
    out = s["base"].double()
    for n in torch.unique(s["row_adapter"]).tolist():
        if n >= 0:
            rows = s["row_adapter"] == n
            both = s["x"][rows].double() @ s["a"][n].double().T
            out[rows] += both @ (s["b"][n].double() * s["scales"][n].double()).T
    return dict(out=out)


def _exact_logprobs(s):
    logits, top, rows = s["logits"], s["top"], []
    for x, given in zip(logits.split(64), s["tokens"].long().split(64)):
        x = x.double()
        logp = torch.log_softmax(x, -1)
        p = logp.exp()
        at = x.gather(1, given[:, None])
        before = torch.arange(x.shape[1], device="cuda")[None] < given[:, None]
        row = dict(logprob=logp.gather(1, given[:, None])[:, 0], rank=(1 + (x > at).sum(-1) + ((x == at) & before).sum(-1)).to(torch.int32),
                   entropy=-(p * logp.clamp(min=-1e300)).sum(-1))
        if top:                             # the largest that is left, the lowest index of equals, `top` times
            left, ids = x.clone().clamp(min=-1e300), []
            for _ in range(top):
                is_top = left == left.max(-1, keepdim=True).values
                ids.append(torch.where(is_top, torch.arange(x.shape[1], device="cuda"), x.shape[1]).min(-1).values)
                left.scatter_(1, ids[-1][:, None], -math.inf)
            ids = torch.stack(ids, 1)
            row["top_ids"], row["top_logprobs"] = ids.to(torch.int32), logp.gather(1, ids)
        rows.append(row)
    return {name: torch.cat([row[name] for row in rows]) for name in rows[0]}


def exact(case, seed):
    s = _case_inputs(case, seed)
    return dict(shared=_exact_shared, adapters=_exact_adapters, logprobs=_exact_logprobs)[case["kind"]](s)


# ------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "shared":
        groups, shared, total = _batch(case)
        held = sum(p for _, _, p in groups) + sum(t - p for t, p in zip(total, shared))
        return dict(bytes=held * case["Hkv"] * 2 * (D // 2 + 4) + 4 * len(total) * case["H"] * D, flops=4.0 * sum(total) * case["H"] * D)
    if kind == "adapters":
        M, N, K, r = case["M"], case["N"], case["K"], case["rank"]
        return dict(bytes=2 * (M * K + 2 * M * N + min(case["used"], M) * r * (N + K)), flops=2.0 * M * r * (N + K))
    M, V, top = case["M"], case["V"], case["top"]
    return dict(bytes=M * V * (4 if case["wide"] else 2) + M * (16 + 8 * top), flops=6.0 * M * V)
