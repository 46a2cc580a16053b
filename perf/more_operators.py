"""A decoding step around the 8-bit cache: queries and keys normed and rotated, attention of
many requests over a prefix that they share, and the next tokens drawn.

A case is a dict of plain values.  ``op`` names the entry point:
  rope    kvx.norm_rope       RMS norm of every query and key head with the position rotation
  prefix  kvx.attend_prefix8  attention over shared prefixes and the requests' own tokens
  sample  kvx.sample_tokens   temperature, top-k, top-p, min-p from given random numbers
``H`` KV heads, ``G`` query heads for each of them, head dimension ``d``.  rope: ``T`` rows;
``packed``: queries and keys are parts of one projection's rows; positions up to ``pos``, one
after another where ``run``.  prefix: ``S`` prefixes of pre_lo .. pre_hi tokens, ``B`` requests
spread over them that hold old_lo .. old_hi tokens of their own and bring new_lo .. new_hi new
ones, pages of ``P`` tokens.  sample: ``B`` rows of ``V`` logits, settings of each row by ``mix``.
What ``pick`` draws (lengths, settings) is the same for every seed.
"""

import math
import random

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-6


def _rope(T, H=8, G=8, d=128, dtype="bf16", style=0, factor=1.0, packed=True, run=False, pos=131072,
          name=None):
    c = dict(op="rope", T=T, H=H, G=G, d=d, dtype=dtype, style=style, factor=factor, packed=packed,
             run=run, pos=pos)
    return c if name is None else dict(c, name=name)


def _prefix(S, B, H=8, G=8, d=128, P=16, pre=(0, 0), old=(0, 0), new=(1, 1), dtype="bf16", pick=1,
            name=None):
    c = dict(op="prefix", S=S, B=B, H=H, G=G, d=d, P=P, pre_lo=pre[0], pre_hi=pre[1], old_lo=old[0],
             old_hi=old[1], new_lo=new[0], new_hi=new[1], dtype=dtype, pick=pick)
    return c if name is None else dict(c, name=name)


def _sample(B, V, dtype="f32", mix="nucleus", masked=False, pick=1, name=None):
    c = dict(op="sample", B=B, V=V, dtype=dtype, mix=mix, masked=masked, pick=pick)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # a decoding step of 16 requests, queries and keys where the projection left them: latency
        _rope(16, G=5, name="rope_step"),
        # the toy models' new turn in fp32, interleaved planes
        _rope(333, H=2, G=2, d=64, dtype="f32", style=1, packed=False, run=True, pos=8192, name="rope_f32"),
        # a long prompt, scaled frequencies
        _rope(8192, factor=8.0, run=True, name="rope_prompt"),
        # five continuations of one conversation that have just begun
        _prefix(1, 5, G=5, pre=(5332, 5332), old=(0, 63), pick=2, name="prefix_one"),
        # a decoding step of a full batch after one common context
        _prefix(1, 64, pre=(8191, 8191), old=(1, 1023), pick=3, name="prefix_step"),
        # several contexts of very different length, drafted tokens, head dimension 64
        _prefix(6, 48, G=4, d=64, P=32, pre=(17, 30000), old=(1, 2000), new=(1, 5), pick=4,
                name="prefix_groups"),
        # the toy model in fp32
        _prefix(2, 5, H=2, G=2, d=64, P=32, pre=(31, 251), old=(0, 120), new=(1, 7), dtype="f32", pick=5,
                name="prefix_f32"),
        # questions of different users over one handed-over document, prefilled together
        _prefix(1, 8, P=64, pre=(8192, 8192), new=(64, 400), pick=6, name="prefix_chunk"),
        # the next token of one conversation: latency
        _sample(1, 131072, name="sample_one"),
        # a batch of requests with settings of their own, an odd vocabulary
        _sample(64, 128257, dtype="bf16", mix="each", pick=2, name="sample_step"),
        # high temperatures, tens of thousands of tokens stay in the draw
        _sample(16, 150001, mix="flat", pick=3, name="sample_flat"),
        # a large batch with common settings
        _sample(512, 131072, pick=4, name="sample_batch"),
    ]


def _log_int(rng, lo, hi):
    if lo >= hi:
        return lo
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(max(lo, 0.5)), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rope", "rope", "prefix", "prefix", "prefix", "sample", "sample", "sample"])
    H, G, d = rng.choice([1, 2, 3, 4, 8, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8, 8, 16]), rng.choice([64, 128, 128])
    dtype, pick = rng.choice(["bf16", "bf16", "bf16", "f32"]), rng.randrange(1 << 20)
    if op == "rope":
        most = 8192 * 72 * 128 * 2 // (H * (G + 1) * d * (4 if dtype == "f32" else 2))
        return _rope(_log_int(rng, 1, min(32768, most)), H=H, G=G, d=d, dtype=dtype, style=rng.choice([0, 0, 1]),
                     factor=rng.choice([1.0, 8.0]), packed=rng.choice([True, False]),
                     run=rng.choice([True, False]), pos=_log_int(rng, 1, 131072))
    if op == "sample":
        B = _log_int(rng, 1, 512)
        return _sample(B, _log_int(rng, 100, 160000 if B < 400 else 131072), dtype=rng.choice(["bf16", "f32"]),
                       mix=rng.choice(["nucleus", "each", "each", "flat"]),
                       masked=rng.choice([False, False, True]), pick=pick)
    B = _log_int(rng, 1, 128)
    kind = rng.choice(["step", "step", "draft", "chunk"])
    new_hi = {"step": 1, "draft": rng.randint(2, 8), "chunk": _log_int(rng, 16, 512)}[kind]
    while B * new_hi * H * G > 2 ** 17:                  # query rows
        new_hi = new_hi // 2
    pre_hi, old_hi = _log_int(rng, 1, 65536), _log_int(rng, 1, 4096)
    pairs = 2 ** 29 if dtype == "bf16" else 2 ** 26      # padded pairs of a query row and a key
    while B * new_hi * H * G * (pre_hi + old_hi + new_hi) > pairs and pre_hi > 16:
        pre_hi, old_hi = pre_hi // 2, old_hi // 2 + 1
    while B * new_hi * H * G * (pre_hi + old_hi + new_hi) > pairs and B > 1:
        B = B // 2
    S = rng.randint(1, min(8, B))
    while B * H * d * old_hi > 2 ** 25:                  # bytes of the requests' own keys
        old_hi = old_hi // 2
    while S * H * d * pre_hi > 2 ** 26:                  # and of the prefixes'
        pre_hi = pre_hi // 2
    return _prefix(S, B, H=H, G=G, d=d, P=rng.choice([16, 16, 32, 64, 128]),
                   pre=(rng.choice([0, 1, pre_hi]), pre_hi), old=(0, old_hi),
                   new=(rng.choice([1, new_hi]), new_hi), dtype=dtype, pick=pick)


def _pages(n, P):
    return -(-n // P)


def _lengths(case):
    """Tokens of each prefix, its requests' number, tokens held and new tokens of each request."""
    rng = random.Random(case["pick"])
    S, B = case["S"], case["B"]
    pre = [_log_int(rng, case["pre_lo"], case["pre_hi"]) for _ in range(S)]
    old = [_log_int(rng, case["old_lo"], case["old_hi"]) for _ in range(B)]
    new = [_log_int(rng, case["new_lo"], case["new_hi"]) for _ in range(B)]
    pre[-1] = case["pre_hi"]      # the longest one is always there
    count = [0] * S
    for _ in range(B):
        count[rng.randrange(S)] += 1
    return pre, count, old, new


# What the rows of a batch are drawn with: temperature, top-k, top-p, min-p (off: 0, 1, 0).
_SETTINGS = {
    "nucleus": [(0.7, 50, 0.9, 0.0), (0.8, 40, 0.95, 0.0), (1.0, 100, 0.9, 0.0)],
    "each": [(0.0, 0, 1.0, 0.0), (0.7, 50, 0.9, 0.0), (1.0, 0, 1.0, 0.0), (0.8, 0, 0.95, 0.0), (0.9, 20, 1.0, 0.0),
             (1.2, 0, 1.0, 0.05), (0.6, 1000, 0.8, 0.01), (1.0, 1, 1.0, 0.0)],
    "flat": [(1.5, 0, 0.95, 0.0), (2.0, 0, 1.0, 0.0), (1.8, 20000, 0.99, 0.0), (2.0, 0, 0.9, 0.001)],
}


def _rope_dict(case):
    return dict(theta=5e5 if case["factor"] > 1 else 1e6, style=case["style"], factor=case["factor"],
                low_freq_factor=1.0, high_freq_factor=4.0, original_max_pos=8192)


def _frequencies(case):
    """Turning rate of each plane, float64."""
    r, d = _rope_dict(case), case["d"]
    w = []
    for j in range(d // 2):
        f = r["theta"] ** (-2.0 * j / d)
        if r["factor"] > 1:
            c = r["original_max_pos"] / (2 * math.pi / f)      # turns over the original context
            if c < r["low_freq_factor"]:
                f /= r["factor"]
            elif c <= r["high_freq_factor"]:
                s = (c - r["low_freq_factor"]) / (r["high_freq_factor"] - r["low_freq_factor"])
                f = (1 - s) * f / r["factor"] + s * f
        w.append(f)
    return w


def _cached_rows(shape, g, dev):
    """Cached rows: a few large key channels for each head, as trained models have them."""
    x = torch.randn(shape, generator=g, device=dev)
    big = torch.rand(shape[:-2] + (1, shape[-1]), generator=g, device=dev) < 4 / shape[-1]
    return torch.where(big, 10 * x, x)


def _prepare_rope(case, g, dev):
    T, H, G, d, dt = case["T"], case["H"], case["G"], case["d"], _DTYPES[case["dtype"]]
    x = torch.randn((T, H * (G + 2), d), generator=g, device=dev) * 3
    x = (x * torch.exp(torch.randn((H * (G + 2), d), generator=g, device=dev) * 0.5)).to(dt)
    q, k = x[:, :H * G], x[:, H * G:H * (G + 1)]
    if not case["packed"]:
        q, k = q.contiguous(), k.contiguous()
    qw, kw = (torch.exp(torch.randn(d, generator=g, device=dev) * 0.3).to(dt) for _ in range(2))
    if case["run"]:
        first = int(torch.randint(0, max(case["pos"] - T, 0) + 1, (1,), generator=g, device=dev))
        pos = first + torch.arange(T, device=dev)
    else:
        pos = torch.randint(0, case["pos"], (T,), generator=g, device=dev)
    return dict(case=case, q=q, k=k, qw=qw, kw=kw, rope=_rope_dict(case), pos=pos.to(torch.int32),
                w=torch.tensor(_frequencies(case), dtype=torch.float64, device=dev))


def _prepare_prefix(case, seed, g, dev):
    H, G, d, P, dt = case["H"], case["G"], case["d"], case["P"], _DTYPES[case["dtype"]]
    pre, count, old, new = _lengths(case)
    lens = [o + n for o, n in zip(old, new)]
    used = sum(_pages(n, P) for n in pre + lens)
    N = used + used // 8 + 4
    perm = torch.randperm(N, generator=torch.Generator().manual_seed(seed)).to(torch.int32)

    def tables(lengths, first):
        counts = torch.tensor([_pages(n, P) for n in lengths])
        width = max(int(counts.max()) + 2, 1)
        starts = first + torch.cumsum(counts, 0) - counts
        col = torch.arange(width)
        return torch.where(col < counts[:, None], perm[(starts[:, None] + col).clamp(max=N - 1)],
                           -1).to(torch.int32).to(dev)

    def sums(x):
        return torch.tensor([0] + list(np.cumsum(x)), dtype=torch.int32, device=dev)

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=dev)

    pool = torch.empty((2 * H, N, P, d), dtype=torch.uint8, device=dev)
    scales = torch.empty((2 * H, N), dtype=torch.float32, device=dev)
    for n in range(2 * H):
        x = _cached_rows((N, P, d), g, dev)
        m, e = torch.frexp(x.abs().amax((1, 2)))       # the smallest power of two s with |x| <= 448 s
        scales[n] = torch.ldexp(torch.ones_like(m), e - torch.where(m > 0.875, 8, 9))
        pool[n] = (x / scales[n][:, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    T = sum(new)
    cu = sums(new)
    requests = [0] + [int(x) for x in np.cumsum(count)]
    at = [0] + [int(x) for x in np.cumsum(new)]
    return dict(case=case, pool=pool.view(2, H, N * P, d).view(torch.float8_e4m3fn), scales=scales.view(2, H, N),
                prefix_tables=tables(pre, 0), prefix_lens=ints(pre), prefix_cu=ints(requests),
                tables=tables(lens, sum(_pages(n, P) for n in pre)), lens=ints(lens), cu=cu,
                q=torch.randn((T, H * G, d), generator=g, device=dev).to(dt),
                # what the host knows of the batch: rows of each prefix's requests, longest ones
                rows=[(at[a], at[b]) for a, b in zip(requests, requests[1:])], pre=pre, longest=max(lens),
                most_new=max(new))


def _prepare_sample(case, g, dev):
    B, V = case["B"], case["V"]
    rng = random.Random(case["pick"])
    rows = [rng.choice(_SETTINGS[case["mix"]]) for _ in range(B)]
    x = torch.randn((B, V), generator=g, device=dev)
    x *= 1.5 + torch.rand((B, 1), generator=g, device=dev)
    # a model's few plausible continuations, of very different certainty from row to row
    n = min(V, 64)
    at = torch.randint(0, V, (B, n), generator=g, device=dev)
    lift = torch.rand((B, n), generator=g, device=dev).pow(2) * (4 + 14 * torch.rand((B, 1), generator=g, device=dev))
    x.scatter_add_(1, at, lift)
    if case["masked"]:      # a grammar allows one token in ten
        x.masked_fill_(torch.rand((B, V), generator=g, device=dev) < 0.9, -math.inf)
        x.scatter_(1, at[:, :1], torch.zeros((B, 1), device=dev))
    t, k, p, m = zip(*rows)
    return dict(case=case, logits=x.to(_DTYPES[case["dtype"]]),
                u=torch.rand(B, generator=g, device=dev),
                temperature=torch.tensor(t, device=dev), top_k=torch.tensor(k, dtype=torch.int32, device=dev),
                top_p=torch.tensor(p, device=dev), min_p=torch.tensor(m, device=dev))


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(seed)
    if case["op"] == "rope":
        return _prepare_rope(case, g, dev)
    if case["op"] == "prefix":
        return _prepare_prefix(case, seed, g, dev)
    return _prepare_sample(case, g, dev)


# ---- plain forms ----

def _rope_plain(s):
    c = s["case"]
    angle = s["pos"].double()[:, None] * s["w"]
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    half = c["d"] // 2
    out = []
    for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
        x = x.float()
        x = x * (1 / torch.sqrt((x * x).mean(2, keepdim=True) + _EPS)) * w.float()
        a, b = (x[..., :half], x[..., half:]) if c["style"] == 0 else (x[..., 0::2], x[..., 1::2])
        a, b = a * cos - b * sin, b * cos + a * sin
        x = torch.cat([a, b], 2) if c["style"] == 0 else torch.stack([a, b], 3).flatten(2)
        out.append(x.to(s["q"].dtype))
    return dict(q=out[0], k=out[1])


def _values(s, slot, page):
    """Keys and values of slots in fp32 [2, H, *slot.shape, d]."""
    kv = s["pool"].view(torch.uint8)[:, :, slot].view(torch.float8_e4m3fn).float()
    return kv * s["scales"][:, :, page][..., None]


def _prefix_plain(s):
    c = s["case"]
    B, H, G, d, P = c["B"], c["H"], c["G"], c["d"], c["P"]
    T, dev = s["q"].shape[0], s["q"].device
    n, m, by = s["longest"], s["most_new"], 1 / math.sqrt(d)
    lens, cu = s["lens"].long(), s["cu"].long()
    key = torch.arange(n, device=dev)
    page = torch.where(key < lens[:, None], s["tables"][:, key // P].long(), 0)
    kv = _values(s, page * P + key % P, page)                               # [2, H, B, n, d]
    i = torch.arange(m, device=dev)
    row = (cu[:-1, None] + i).clamp(max=T - 1)                              # [B, m]
    q = s["q"].float().view(T, H, G, d)
    x = q[row].permute(2, 0, 3, 1, 4).reshape(H, B, G * m, d)
    score = torch.matmul(x, kv[0].transpose(2, 3).contiguous()).view(H, B, G, m, n) * by
    last = lens[:, None] - (cu[1:] - cu[:-1])[:, None] + i                  # a row's own position
    score = torch.where((key <= last[:, :, None])[None, :, None], score, -math.inf)
    t = torch.arange(T, device=dev)
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    out, lse = torch.empty((T, H, G, d), device=dev), torch.empty((T, H, G), device=dev)
    for share, (t0, t1) in enumerate(s["rows"]):
        if t0 == t1:
            continue
        bs, rows = b[t0:t1], t[t0:t1] - cu[b[t0:t1]]
        mine = score[:, bs, :, rows].permute(1, 0, 2, 3)      # [H, rows, G, n]
        key_p = torch.arange(s["pre"][share], device=dev)
        page_p = s["prefix_tables"][share, key_p // P].long()
        kp, vp = _values(s, page_p * P + key_p % P, page_p)                 # [H, keys, d]
        xq = q[t0:t1].transpose(0, 1).reshape(H, (t1 - t0) * G, d)
        common = (torch.matmul(xq, kp.transpose(1, 2).contiguous()) * by).view(H, t1 - t0, G, len(key_p))
        top = mine.amax(3)
        if len(key_p):
            top = torch.maximum(top, common.amax(3))
        mine, common = torch.exp(mine - top[..., None]), torch.exp(common - top[..., None])
        total = mine.sum(3) + common.sum(3)
        o = torch.matmul(common.view(H, (t1 - t0) * G, len(key_p)), vp).view(H, t1 - t0, G, d)
        # a request's rows with its own values
        weights = torch.zeros((H, B, m, G, n), device=dev)
        weights[:, bs, rows] = mine
        ov = torch.matmul(weights.view(H, B, m * G, n), kv[1]).view(H, B, m, G, d)
        o = (o + ov[:, bs, rows]) / total[..., None]
        out[t0:t1] = o.transpose(0, 1)
        lse[t0:t1] = (top + torch.log(total)).transpose(0, 1)
    return dict(out=out.reshape(T, H * G, d).to(s["q"].dtype), lse=lse.reshape(T, H * G))


def _sample_plain(s):
    x = s["logits"].float()
    B, V = x.shape
    at = torch.arange(V, device=x.device)
    top = x.amax(1, keepdim=True)
    first = torch.where(x == top, at, V).amin(1)
    t = s["temperature"].double()[:, None]
    w = torch.exp((x.double() - top.double()) / torch.where(t > 0, t, 1.0))
    value, order = torch.sort(x, dim=1, descending=True, stable=True)         # equal ones by index
    ranked = w.gather(1, order)
    k = s["top_k"].long()[:, None]
    keep = (at < k) | (k <= 0)
    cum = torch.cumsum(ranked * keep, 1)
    p = s["top_p"].double()[:, None]
    keep &= (cum - ranked < p * cum[:, -1:]) | (p >= 1) | (at == 0)
    keep &= ranked >= s["min_p"].double()[:, None]
    w = w * torch.zeros_like(keep).scatter_(1, order, keep)
    cum = torch.cumsum(w, 1)
    total = cum[:, -1]
    token = (cum <= s["u"].double()[:, None] * total[:, None]).sum(1).clamp(max=V - 1)
    greedy = s["temperature"] <= 0
    token = torch.where(greedy, first, token)
    logprob = torch.log(w.gather(1, token[:, None])[:, 0] / total)
    return dict(tokens=token.to(torch.int32), logprob=torch.where(greedy, 0.0, logprob).float())


def run(s):
    op = s["case"]["op"]
    if not own:
        return {"rope": _rope_plain, "prefix": _prefix_plain, "sample": _sample_plain}[op](s)
    from paper_2608_03893_amd import kvx
    if op == "rope":
        q, k = kvx.norm_rope(s["q"], s["k"], s["qw"], s["kw"], s["rope"], s["pos"], eps=_EPS)
        return dict(q=q, k=k)
    if op == "prefix":
        if "workspace" not in s:      # kept from step to step
            s["workspace"] = kvx.prefix_workspace(s["q"], s["pool"], s["prefix_tables"], s["tables"])
        out, lse = kvx.attend_prefix8(s["q"], s["pool"], s["scales"], s["prefix_tables"], s["prefix_lens"],
                                      s["prefix_cu"], s["tables"], s["lens"], s["cu"], with_lse=True,
                                      workspace=s["workspace"])
        return dict(out=out, lse=lse)
    if "workspace" not in s:
        s["workspace"] = kvx.sample_workspace(s["logits"])
    tokens, logprob = kvx.sample_tokens(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"],
                                        with_logprob=True, workspace=s["workspace"])
    return dict(tokens=tokens, logprob=logprob)


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "sample":
        B, V = case["B"], case["V"]
        return dict(bytes=B * V * e + B * 28, flops=B * V)
    H, G, d = case["H"], case["G"], case["d"]
    if case["op"] == "rope":
        n = case["T"] * H * (G + 1) * d
        # squares and their sum, two factors, three operations of the rotation
        return dict(bytes=2 * n * e + 4 * case["T"] + 2 * d * e, flops=7 * n)
    pre, count, old, new = _lengths(case)
    P, T = case["P"], sum(new)
    cu = [0] + [int(x) for x in np.cumsum(count)]
    lens = [o + n for o, n in zip(old, new)]
    keys = sum(n for n, m in zip(pre, count) if m) + sum(lens)
    pages = sum(_pages(n, P) for n, m in zip(pre, count) if m) + sum(_pages(n, P) for n in lens)
    pairs = sum(n * o + n * (n + 1) // 2 for o, n in zip(old, new))
    pairs += sum(n * sum(new[a:b]) for n, a, b in zip(pre, cu, cu[1:]))
    return dict(bytes=2 * H * (keys * d + pages * 4) + 4 * pages + T * H * G * (2 * d * e + 4),
                flops=4 * d * H * G * pairs)


# ---- the operators' definitions in 64 bits ----

def _exact_rope(s):
    c = s["case"]
    angle = s["pos"].double()[:, None] * s["w"]
    turn = torch.complex(torch.cos(angle), torch.sin(angle))[:, None]
    out = []
    for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])):
        x = x.double()
        x = x / torch.sqrt((x ** 2).sum(2, keepdim=True) / c["d"] + _EPS) * w.double()
        if c["style"] == 0:
            z = torch.complex(*[h.contiguous() for h in x.chunk(2, 2)]) * turn
            out.append(torch.cat([z.real, z.imag], 2))
        else:
            z = torch.view_as_complex(x.view(x.shape[:2] + (-1, 2)).contiguous()) * turn
            out.append(torch.view_as_real(z).flatten(2))
    return dict(q=out[0], k=out[1])


def _exact_prefix(s):
    c = s["case"]
    H, G, d, P = c["H"], c["G"], c["d"], c["P"]
    T, dev = s["q"].shape[0], s["q"].device
    out = torch.zeros((T, H * G, d), dtype=torch.float64, device=dev)
    lse = torch.full((T, H * G), -math.inf, dtype=torch.float64, device=dev)
    cu, lens, shares = s["cu"].tolist(), s["lens"].tolist(), s["prefix_cu"].tolist()
    for b in range(c["B"]):
        a, z = cu[b], cu[b + 1]
        share = max(i for i in range(c["S"]) if shares[i] <= b)
        n0, n1 = s["pre"][share], lens[b]
        hidden = torch.arange(n0 + n1, device=dev) > n0 + n1 - (z - a) + torch.arange(z - a, device=dev)[:, None]
        pages = torch.cat([s["prefix_tables"][share, :_pages(n0, P)], s["tables"][b, :_pages(n1, P)]]).long()
        held = torch.cat([torch.arange(n0, device=dev), _pages(n0, P) * P + torch.arange(n1, device=dev)])
        for h in range(H):
            k, v = ((s["pool"][i, h].view(torch.uint8).view(-1, P, d)[pages].view(torch.float8_e4m3fn).float().double()
                     * s["scales"][i, h, pages].double()[:, None, None]).view(-1, d)[held] for i in range(2))
            for q in range(h * G, (h + 1) * G):
                x = (s["q"][a:z, q].double() @ k.t()) / math.sqrt(d)
                x.masked_fill_(hidden, -math.inf)
                lse[a:z, q] = torch.logsumexp(x, 1)
                out[a:z, q] = torch.softmax(x, 1) @ v
    return dict(out=out, lse=lse)


def _exact_sample(s):
    x = s["logits"].double().cpu().numpy()
    u, temperature, top_k, top_p, min_p = (s[n].double().cpu().numpy()
                                           for n in ("u", "temperature", "top_k", "top_p", "min_p"))
    tokens, logprob = np.zeros(len(x), np.int32), np.zeros(len(x))
    for b, row in enumerate(x):
        best = int(np.argmax(row))
        tokens[b] = best
        if temperature[b] <= 0:
            continue
        # tokens of less than 1e-20 of the best one's weight are nobody's
        some = np.flatnonzero(row >= row[best] - 46 * temperature[b])
        weight = np.exp((row[some] - row[best]) / temperature[b])
        order = np.argsort(-row[some], kind="stable")
        if top_k[b] > 0:
            order = order[:int(top_k[b])]
        if top_p[b] < 1:
            cum = np.cumsum(weight[order])
            order = order[:max(int(np.searchsorted(cum, top_p[b] * cum[-1])) + 1, 1)]
        order = order[weight[order] >= min_p[b]]
        kept = np.sort(order)
        cum = np.cumsum(weight[kept])
        n = min(int(np.searchsorted(cum, u[b] * cum[-1], side="right")), len(kept) - 1)
        tokens[b], logprob[b] = some[kept[n]], math.log(weight[kept[n]] / cum[-1])
    dev = s["logits"].device
    return dict(tokens=torch.tensor(tokens, device=dev), logprob=torch.tensor(logprob, device=dev))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rope(s)
    if case["op"] == "prefix":
        # a request's heads one by one: too many of them take too long
        return _exact_prefix(s) if case["B"] * case["H"] * case["G"] <= 20000 else None
    return _exact_sample(s)
