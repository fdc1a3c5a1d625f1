"""The operators that a serving program runs between the QKV projection and the output projection when its 4-bit KV cache is
paged, each in its plain form and as the framework's call:

  append   queries and keys of new tokens: optional RMSNorm of every head and the position rotation; keys and values quantized
           to 4 bits into the pages of their sequences.  The tokens just written are read back, as the values they stand for.
  gather   tokens of the paged cache as FP16 keys and values, for a prompt that goes on behind a cached prefix
  decode   attention of one new token per sequence over the paged cache, whole or through a sliding window with first tokens
           that stay visible (sinks)
  prefill  causal attention over ragged prompts, whole or through such a window, new tokens at the end of the keys

Heads are those of the models that the benchmark measures, and generic ones.  Sequence lengths of a case run evenly from its
longest down to half of it.  The plain forms hold the same cache as arrays: two codes to a byte, scales and zeros beside them.
"""
import math

import torch

own = False

D = 128                     # head dimension
PAGE = 64                   # tokens of a page
EPS = 1e-6


# ------------------------------------------------------------------------------------------------------------------
# The cases
# ------------------------------------------------------------------------------------------------------------------
def listed():
    return [
        # generation for one user, multi-head attention: launches and latency only
        dict(name="append-1x1-h32-32", kind="append", H=32, Hkv=32, B=1, tokens=1, cached=1022, norm=False, rot=128, near=False),
        # a full batch of a grouped-query model with norms of queries and keys
        dict(name="append-64x1-h32-8-norm", kind="append", H=32, Hkv=8, B=64, tokens=1, cached=1500, norm=True, rot=128, near=False),
        # five ragged prompts of the largest model behind a shared prefix that ends inside a page
        dict(name="append-5x1733-h64-8", kind="append", H=64, Hkv=8, B=5, tokens=1733, cached=77, norm=False, rot=128, near=False),
        # one short cached prefix that its prompt goes on behind
        dict(name="gather-1x389-h32", kind="gather", Hkv=32, B=1, tokens=389),
        # prefixes of a batch of long conversations
        dict(name="gather-6x6000-h8", kind="gather", Hkv=8, B=6, tokens=6000),
        # generation for one user far into a conversation: few pairs of a sequence and a KV head, the length is cut
        dict(name="decode-1x8192-h32-8", kind="decode", H=32, Hkv=8, B=1, context=8192, window=0, sinks=0),
        # a full batch of a multi-head model: the cache's bytes
        dict(name="decode-64x1024-h32-32", kind="decode", H=32, Hkv=32, B=64, context=1024, window=0, sinks=0),
        # an ordinary batch on the largest model, ragged
        dict(name="decode-37x700-h64-8", kind="decode", H=64, Hkv=8, B=37, context=700, window=0, sinks=0),
        # long conversations through a window of 4096 tokens and four sinks
        dict(name="decode-16x32000-h32-8-window", kind="decode", H=32, Hkv=8, B=16, context=32000, window=4096, sinks=4),
        # one ordinary prompt
        dict(name="prefill-1x1024-h32-32", kind="prefill", H=32, Hkv=32, B=1, tokens=1024, cached=0, window=0, sinks=0),
        # ragged prompts on the largest model: the most work in one pass
        dict(name="prefill-3x4001-h64-8", kind="prefill", H=64, Hkv=8, B=3, tokens=4001, cached=0, window=0, sinks=0),
        # a chunk of a long prompt behind what is cached already, through a window with sinks
        dict(name="prefill-1x2048-after-6100-h32-8-window", kind="prefill", H=32, Hkv=8, B=1, tokens=2048, cached=6100, window=1024, sinks=4),
    ]


_HEADS = ((32, 32), (32, 8), (64, 8), (28, 4), (40, 8), (16, 1), (9, 3))


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(("append", "gather", "decode", "decode", "prefill", "prefill"))
    H, Hkv = rng.choice(_HEADS)
    if kind == "append":
        if rng.random() < 0.5:
            B, tokens = _log_int(rng, 1, 256), 1
        else:
            B = _log_int(rng, 1, 16)
            tokens = _log_int(rng, 2, 1000000 // (B * (2 * H + 3 * Hkv)))
        return dict(kind=kind, H=H, Hkv=Hkv, B=B, tokens=tokens, cached=rng.randint(0, 5000), norm=rng.random() < 0.5,
                    rot=rng.choice((128, 128, 64)), near=rng.random() < 0.3)
    if kind == "gather":
        B = _log_int(rng, 1, 32)
        return dict(kind=kind, Hkv=Hkv, B=B, tokens=_log_int(rng, 1, min(32768, 200000 // (B * Hkv))))
    if kind == "decode":
        B = _log_int(rng, 1, 128)
        context = _log_int(rng, 1, min(32768, 64 * 1024 * 32 // (B * Hkv)))
        window = rng.choice((0, _log_int(rng, 1, 4096)))
        return dict(kind=kind, H=H, Hkv=Hkv, B=B, context=context, window=window, sinks=rng.choice((0, 4, 70)) if window else 0)
    B = _log_int(rng, 1, 8)
    tokens = _log_int(rng, 1, 4001 // B)
    cached = rng.choice((0, rng.randint(1, max(1, min(6000, 900000000 // (H * B * tokens) - tokens // 2)))))
    window = rng.choice((0, _log_int(rng, 1, 2048)))
    return dict(kind=kind, H=H, Hkv=Hkv, B=B, tokens=tokens, cached=cached, window=window, sinks=rng.choice((0, 4, 70)) if window else 0)


def _lengths(B, longest):
    """B lengths from `longest` down to half of it."""
    return [longest - (longest // 2) * b // max(B - 1, 1) for b in range(B)]


def _starts(case):
    """What each sequence of a case holds already: evenly from `cached` down to half of it."""
    return _lengths(case["B"], case["cached"])


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


def _ints(values, device):
    return torch.tensor(values, dtype=torch.int32, device=device)


def _cumulative(lengths):
    total, out = 0, [0]
    for n in lengths:
        total += n
        out.append(total)
    return out


def _tables(g, totals):
    """A block table whose sequences' pages lie anywhere in the pool, and the number of pages of that pool."""
    need = [-(-max(t, 1) // PAGE) for t in totals]
    width, pages = max(need), sum(need) + 3
    perm = torch.randperm(pages, generator=g, device=g.device).to(torch.int32)
    at = _cumulative(need)
    table = torch.full((len(totals), width), -1, dtype=torch.int32, device=g.device)
    for b, n in enumerate(need):
        table[b, :n] = perm[at[b]:at[b] + n]
    return table, pages


def _angles(rows, rot, device):
    """FP32 table [rows, rot]: cosines, then sines, of position x 10000^(-2 i / rot)."""
    inv = 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    a = torch.arange(rows, dtype=torch.float64, device=device)[:, None] * inv
    return torch.cat((a.cos(), a.sin()), dim=1).to(torch.float32)


def _case_inputs(case, seed):
    """What the plain form, the framework's calls and the exact form start from."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    kind, B, Hkv = case["kind"], case["B"], case["Hkv"]
    s = dict(case)
    if kind == "append":
        H, starts, new = case["H"], _starts(case), _lengths(B, case["tokens"])
        M = sum(new)
        s["table"], s["pages"] = _tables(g, [a + n for a, n in zip(starts, new)])
        qkv = _normal(g, M, H + 2 * Hkv, D)
        qkv[:, H:H + Hkv] = _keys(g, M, Hkv, D)
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        s["cu"], s["starts"] = _ints(_cumulative(new), "cuda"), _ints(starts, "cuda")
        s["angles"] = _angles(max(a + n for a, n in zip(starts, new)), case["rot"], "cuda")
        s["gq"] = 1.0 + 0.1 * _normal(g, D) if case["norm"] else None
        s["gk"] = 1.0 + 0.1 * _normal(g, D) if case["norm"] else None
        return s
    if kind == "prefill":
        H, new, held = case["H"], _lengths(B, case["tokens"]), _starts(case)
        total = [n + h for n, h in zip(new, held)]
        M, Mk = sum(new), sum(total)
        s["q"] = _normal(g, M, H, D)
        if case["cached"]:                  # keys and values gathered from the cache
            s["k"], s["v"] = _keys(g, Mk, Hkv, D), _normal(g, Mk, Hkv, D)
        else:                               # keys rotated into a tensor of their own, values where the projection left them
            s["k"], s["v"] = _keys(g, Mk, Hkv, D), _normal(g, Mk, H + 2 * Hkv, D)[:, H + Hkv:]
        s["cu_q"], s["cu_k"] = _ints(_cumulative(new), "cuda"), _ints(_cumulative(total), "cuda")
        return s
    lens = _lengths(B, case["tokens"] if kind == "gather" else case["context"])
    if kind == "decode" and B >= 8:
        lens[-1] = 0                        # a slot of the batch that no request holds
    M = sum(lens)
    s["table"], s["pages"] = _tables(g, lens)
    s["cu"], s["starts"], s["lens"] = _ints(_cumulative(lens), "cuda"), _ints([0] * B, "cuda"), _ints(lens, "cuda")
    s["k"], s["v"] = _keys(g, M, Hkv, D), _normal(g, M, Hkv, D)
    if kind == "decode":
        s["q"] = _normal(g, B, case["H"], D)
    return s


def prepare(case, seed):
    s = _case_inputs(case, seed)
    kind, B, Hkv = s["kind"], s["B"], s["Hkv"]
    if kind == "prefill":
        if own:
            from paper_2405_04532_amd import api
            need = api.attention_prefill_workspace_bytes(s["q"].shape[0], s["k"].shape[0], B, s["H"], Hkv, s["window"], s["sinks"])
            s["workspace"] = api.new_workspace(need, "cuda")
        return s
    if own:
        from paper_2405_04532_amd import api
        s["pool"] = api.kv4_new_pool(s["pages"], Hkv, "cuda")
        if kind != "append":
            api.kv4_paged_append(s["pool"], s["k"], s["v"], s["table"], s["cu"], s["starts"])
        if kind == "decode":
            need = api.kv4_paged_attention_workspace_bytes(B, s["H"], Hkv, s["table"].shape[1], s["window"], s["sinks"])
            s["workspace"] = api.new_workspace(need, "cuda")
            s["out"] = torch.empty((B, s["H"], D), dtype=torch.float16, device="cuda")
    else:
        s["pool"] = _plain_pool(s["pages"], Hkv, "cuda")
        if kind != "append":
            _plain_write(s["pool"], s["k"], s["v"], s["table"], s["cu"], s["starts"])
    if kind != "append":
        del s["k"], s["v"]                  # the cache holds them
    return s


# ------------------------------------------------------------------------------------------------------------------
# Plain forms
# ------------------------------------------------------------------------------------------------------------------
def _plain_pool(pages, Hkv, device):
    """For keys and for values: two codes to a byte [pages, Hkv, PAGE, D / 2], scales and zeros [pages, Hkv, PAGE]."""
    half = lambda: (torch.zeros((pages, Hkv, PAGE, D // 2), dtype=torch.uint8, device=device),  # noqa: E731
                    torch.zeros((pages, Hkv, PAGE), dtype=torch.float16, device=device),
                    torch.zeros((pages, Hkv, PAGE), dtype=torch.float16, device=device))
    return half(), half()


def _token_of_row(cu, starts, rows):
    """Sequence and position of each row of a ragged batch."""
    row = torch.arange(rows, device=cu.device)
    seq = torch.searchsorted(cu[1:].long(), row, right=True)
    return seq, starts.long()[seq] + row - cu.long()[seq]


def _plain_write(pool, k, v, table, cu, starts):
    seq, pos = _token_of_row(cu, starts, k.shape[0])
    page, off = table[seq, pos // PAGE].long(), pos % PAGE
    _plain_write_half(pool[0], k, page, off)
    _plain_write_half(pool[1], v, page, off)


def _plain_write_half(half, x, page, off):
    """Eq. 1 with four bits; in 64 bits, since codes are decided at half-integers."""
    codes, scale, zero = half
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


def _plain_read(pool, table, cu, starts, rows):
    seq, pos = _token_of_row(cu, starts, rows)
    page, off = table[seq, pos // PAGE].long(), pos % PAGE
    k, v = (_plain_values(c[page, :, off], s[page, :, off], z[page, :, off]).half() for c, s, z in pool)
    return k, v


def _plain_rotate(x, gamma, angles, rot, near):
    """Norm and rotation in 64 bits (the key's codes are decided on the result), rounded once."""
    x = x.double()
    if gamma is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma.double()
    cos, sin = angles[:, None, :rot // 2].double(), angles[:, None, rot // 2:].double()
    r = x[..., :rot]
    if near:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2)
    else:
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat((a * cos - b * sin, b * cos + a * sin), dim=-1)
    return torch.cat((r, x[..., rot:]), dim=-1).half()


def _plain_append(s):
    rows = s["q"].shape[0]
    _, pos = _token_of_row(s["cu"], s["starts"], rows)
    angles = s["angles"][pos]
    q = _plain_rotate(s["q"], s["gq"], angles, s["rot"], s["near"])
    k = _plain_rotate(s["k"], s["gk"], angles, s["rot"], s["near"])
    _plain_write(s["pool"], k, s["v"], s["table"], s["cu"], s["starts"])
    return q, k


def _plain_softmax(score, visible):
    """Softmax over the last axis of what is visible; a row that sees nothing is zero."""
    score = score.masked_fill(~visible, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total > 0, total, torch.ones_like(total))


def _plain_decode(s):
    B, H, Hkv, window, sinks = s["B"], s["H"], s["Hkv"], s["window"], s["sinks"]
    lens, table = s["lens"].long()[:, None], s["table"]
    width = table.shape[1]
    index = torch.arange(width, device=table.device).expand(B, width)
    first = 0
    if window:                              # the pages of the sinks, then those that the window reaches
        first = -(-sinks // PAGE)
        reach = (lens - window).clamp(min=0) // PAGE + torch.arange((window + PAGE - 2) // PAGE + 1, device=table.device)
        index = torch.cat((index[:, :first], torch.where(reach < first, width, reach)), dim=1)
    held = index < width
    page = torch.where(held, table.gather(1, index.clamp(max=width - 1)), 0).long().clamp(min=0)
    t = (index[..., None] * PAGE + torch.arange(PAGE, device=table.device)).flatten(1)
    visible = (t < lens) & held.repeat_interleave(PAGE, 1)
    if window:
        visible &= (t >= lens - window) | (t < sinks)
    k, v = (_plain_values(c[page], z_s[page], z[page]).transpose(1, 2).reshape(B, Hkv, -1, D) for c, z_s, z in s["pool"])
    q = s["q"].float().view(B, Hkv, H // Hkv, D)
    p = _plain_softmax(torch.matmul(q, k.transpose(-1, -2)) / math.sqrt(D), visible[:, None, None])
    return torch.matmul(p, v).view(B, H, D).half()


def _padded(x, cu, longest):
    """Rows of a ragged batch [M, heads, D] as [B, heads, longest, D] in 32 bits."""
    row = cu[:-1].long()[:, None] + torch.arange(longest, device=x.device)
    return x[row.clamp(max=x.shape[0] - 1)].transpose(1, 2).float()


def _plain_prefill(s):
    B, H, Hkv, tokens, window = s["B"], s["H"], s["Hkv"], s["tokens"], s["window"]
    cu_q, cu_k = s["cu_q"].long(), s["cu_k"].long()
    reach = tokens + s["cached"]
    q = _padded(s["q"], cu_q, tokens).reshape(B, Hkv, H // Hkv * tokens, D)
    k, v = _padded(s["k"], cu_k, reach), _padded(s["v"], cu_k, reach)
    n_q, n_k = (cu_q[1:] - cu_q[:-1])[:, None], (cu_k[1:] - cu_k[:-1])[:, None]
    pos = (n_k - n_q + torch.arange(tokens, device=q.device))[..., None]
    t = torch.arange(reach, device=q.device)
    visible = (t <= pos) & (t < n_k[..., None])
    if window:
        visible &= (t > pos - window) | (t < s["sinks"])
    score = torch.matmul(q, k.transpose(-1, -2)).view(B, Hkv, H // Hkv, tokens, reach) / math.sqrt(D)
    p = _plain_softmax(score, visible[:, None, None])
    out = torch.matmul(p.view(B, Hkv, -1, reach), v).view(B, H, tokens, D)
    seq, i = _token_of_row(cu_q, torch.zeros_like(cu_q[1:]), s["q"].shape[0])
    return out[seq, :, i].half()


# ------------------------------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------------------------------
def run(s):
    kind = s["kind"]
    if own:
        from paper_2405_04532_amd import api
        if kind == "append":
            q, k = api.qk_rope_kv4_append(s["q"], s["k"], s["v"], s["pool"], s["table"], s["cu"], s["starts"], s["angles"],
                                          q_gamma=s["gq"], k_gamma=s["gk"], eps=EPS, interleaved=s["near"], want_k=True)
            kc, vc = api.kv4_paged_gather(s["pool"], s["table"], s["cu"], s["starts"], q.shape[0], s["Hkv"])
            return dict(q=q, k=k, cached_k=kc, cached_v=vc)
        if kind == "gather":
            k, v = api.kv4_paged_gather(s["pool"], s["table"], s["cu"], s["starts"], sum(_lengths(s["B"], s["tokens"])), s["Hkv"])
            return dict(k=k, v=v)
        if kind == "decode":
            return dict(out=api.kv4_paged_attention_decode(s["q"], s["pool"], s["table"], s["lens"], s["Hkv"], window=s["window"],
                                                           sinks=s["sinks"], out=s["out"], workspace=s["workspace"]))
        return dict(out=api.attention_prefill(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], window=s["window"], sinks=s["sinks"],
                                              workspace=s["workspace"]))
    if kind == "append":
        q, k = _plain_append(s)
        kc, vc = _plain_read(s["pool"], s["table"], s["cu"], s["starts"], q.shape[0])
        return dict(q=q, k=k, cached_k=kc, cached_v=vc)
    if kind == "gather":
        k, v = _plain_read(s["pool"], s["table"], s["cu"], s["starts"], sum(_lengths(s["B"], s["tokens"])))
        return dict(k=k, v=v)
    return dict(out=_plain_decode(s) if kind == "decode" else _plain_prefill(s))


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


def _exact_turned(x, gamma, position, rot, near):
    """Heads [n, heads, D] at `position` [n]: pairs as complex numbers times those of the FP32 table."""
    y = x.double()
    if gamma is not None:
        y = y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / D + EPS) * gamma.double()
    i = torch.arange(rot // 2, dtype=torch.float64, device=x.device)
    angle = position.double()[:, None] * torch.pow(torch.tensor(10000.0, dtype=torch.float64, device=x.device), -2 * i / rot)
    turn = torch.complex(angle.cos().float().double(), angle.sin().float().double())[:, None]
    part = y[..., :rot].unflatten(-1, (-1, 2)) if near else y[..., :rot].unflatten(-1, (2, -1)).transpose(-1, -2)
    z = torch.view_as_real(torch.complex(part[..., 0].contiguous(), part[..., 1].contiguous()) * turn)
    y = y.clone()
    y[..., :rot] = (z if near else z.transpose(-1, -2)).flatten(-2)
    return y


def _exact_attention(q, k, v, position, window, sinks):
    """q [n, H, D] at `position` [n] over k, v [t, Hkv, D], in 64 bits, a KV head at a time."""
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    t, p = torch.arange(k.shape[0], device=q.device)[None, :], position[:, None]
    seen = t <= p
    if window:
        seen = seen & ((p - t < window) | (t < sinks))
    some, r = seen.any(1), q.shape[1] // k.shape[1]
    for h in range(q.shape[1]):
        a = (q[:, h].double() @ k[:, h // r].double().T) * D ** -0.5
        a = torch.softmax(torch.where(seen, a, torch.full_like(a, -1e300)), dim=1)
        out[:, h] = torch.where(some[:, None], (a * seen) @ v[:, h // r].double(), 0.0)
    return out


def exact(case, seed):
    s = _case_inputs(case, seed)
    kind = case["kind"]
    if kind == "append":
        new, starts = _lengths(case["B"], case["tokens"]), _starts(case)
        at = torch.cat([torch.arange(a, a + n) for a, n in zip(starts, new)]).cuda()
        q = _exact_turned(s["q"], s["gq"], at, case["rot"], case["near"])
        k = _exact_turned(s["k"], s["gk"], at, case["rot"], case["near"])
        return dict(q=q, k=k, cached_k=_exact_cached(k.to(torch.float16)), cached_v=_exact_cached(s["v"]))
    if kind == "gather":
        return dict(k=_exact_cached(s["k"]), v=_exact_cached(s["v"]))
    if kind == "decode":
        cu, out = s["cu"].tolist(), []
        for b in range(case["B"]):
            n = cu[b + 1] - cu[b]
            k, v = _exact_cached(s["k"][cu[b]:cu[b + 1]]), _exact_cached(s["v"][cu[b]:cu[b + 1]])
            last = torch.full((1,), n - 1, device="cuda")
            out.append(_exact_attention(s["q"][b:b + 1], k, v, last, case["window"], case["sinks"]) if n else
                       torch.zeros((1, case["H"], D), dtype=torch.float64, device="cuda"))
        return dict(out=torch.cat(out))
    cu_q, cu_k, out = s["cu_q"].tolist(), s["cu_k"].tolist(), []
    for b in range(case["B"]):
        n, m = cu_q[b + 1] - cu_q[b], cu_k[b + 1] - cu_k[b]
        out.append(_exact_attention(s["q"][cu_q[b]:cu_q[b + 1]], s["k"][cu_k[b]:cu_k[b + 1]], s["v"][cu_k[b]:cu_k[b + 1]],
                                    torch.arange(m - n, m, device="cuda"), case["window"], case["sinks"]))
    return dict(out=torch.cat(out))


# ------------------------------------------------------------------------------------------------------------------
# What a pass cannot do without
# ------------------------------------------------------------------------------------------------------------------
def _seen(length, window, sinks):
    """Tokens that the last of `length` tokens sees."""
    return length if not window or length <= window else window + min(sinks, length - window)


def work(case):
    kind, B, Hkv = case["kind"], case["B"], case["Hkv"]
    cached = 2 * (D // 2 + 4)               # a token's key and value in the cache, of one KV head
    if kind == "append":
        M, H = sum(_lengths(B, case["tokens"])), case["H"]
        moved = M * D * 2 * (2 * H + 3 * Hkv) + M * Hkv * cached + M * Hkv * D * 4 + M * case["rot"] * 4
        return dict(bytes=moved, flops=M * (H + Hkv) * (3 * case["rot"] + (4 * D if case["norm"] else 0)))
    if kind == "gather":
        M = sum(_lengths(B, case["tokens"]))
        return dict(bytes=M * Hkv * (cached + D * 4), flops=M * Hkv * D * 4)
    if kind == "decode":
        lens = _lengths(B, case["context"])
        if B >= 8:
            lens[-1] = 0
        seen = sum(_seen(n, case["window"], case["sinks"]) for n in lens)
        return dict(bytes=seen * Hkv * cached + 4 * B * case["H"] * D, flops=4.0 * seen * case["H"] * D)
    new, held, H = _lengths(B, case["tokens"]), _starts(case), case["H"]
    seen = sum(_seen(h + i + 1, case["window"], case["sinks"]) for n, h in zip(new, held) for i in range(n))
    M, Mk = sum(new), sum(new) + sum(held)
    if case["window"]:                      # keys that some query of the sequence sees
        Mk = sum(min(n + h, n + case["window"] - 1 + case["sinks"]) for n, h in zip(new, held))
    return dict(bytes=(2 * M * H + 2 * Mk * Hkv) * D * 2, flops=4.0 * seen * H * D)
