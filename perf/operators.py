"""Measured cases of the operators of a drafter's decoding step: appending rotated keys and values to a paged cache
(hsd_kv_append), attention of one new token per sequence over that cache (hsd_paged_attention), few-row products with 4-bit
weights (hsd_gemm_w4) and log probabilities of given tokens with entropy, rank and top alternatives (hsd_token_logprobs).

`own` chooses what run() does: the plain forms in elementary torch operations, or the calls of the package."""
import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}
MOST_KEY_BYTES = 1 << 30          # of a drawn cache, below the largest listed one's
MOST_WEIGHTS = 100 << 20          # of a drawn matrix: its plain form writes them out in 32 bits


def listed():
    return [
        # one sequence of the 8B shape after its prompt of 1024 tokens: latency
        dict(name="attention, one sequence", op="attention", dtype="bf16", batch=1, nq=32, nkv=8, hd=128, page=16, longest=1025, ragged=False),
        # the long-context shape: a batch of 16 at 8192 tokens and a few
        dict(name="attention, 16 x 8200", op="attention", dtype="bf16", batch=16, nq=32, nkv=8, hd=128, page=16, longest=8200, ragged=False),
        # serving: many sequences of any length up to 12000
        dict(name="attention, 48 ragged", op="attention", dtype="bf16", batch=48, nq=32, nkv=8, hd=128, page=16, longest=12000, ragged=True),
        # a small fp32 model's heads, a batch of short sequences
        dict(name="attention, fp32 heads of 32", op="attention", dtype="fp32", batch=12, nq=8, nkv=2, hd=32, page=16, longest=700, ragged=True),
        # one drafted token: the projections' fp32 rows into a bf16 cache
        dict(name="append, one token", op="append", source="fp32", dtype="bf16", batch=1, rows=1, nq=32, nkv=8, hd=128, page=16, before=1024),
        # prompts of a batch, ragged, together
        dict(name="append, prompts of 7", op="append", source="bf16", dtype="bf16", batch=7, rows=8191, nq=32, nkv=8, hd=128, page=16, before=300),
        # one token through a square projection
        dict(name="w4, 1 x 4096 x 4096", op="w4", rows=1, N=4096, K=4096, group=128),
        # nine rows (eight drafts and one more) through gate and up of the 8B shape
        dict(name="w4, 9 x 28672 x 4096", op="w4", rows=9, N=28672, K=4096, group=128),
        # a batch through the output head of the 1B shape, small groups
        dict(name="w4, 32 x 32000 x 2048", op="w4", rows=32, N=32000, K=2048, group=32),
        # one sampled token and its alternatives
        dict(name="logprobs, one row", op="logprobs", dtype="bf16", rows=1, V=32000, top=20),
        # the acceptance workload's target rows: 64 sequences of nine
        dict(name="logprobs, 576 rows", op="logprobs", dtype="bf16", rows=576, V=32000, top=5),
        # scores of a text under a large vocabulary
        dict(name="logprobs, 700 x 131072", op="logprobs", dtype="fp32", rows=700, V=131072, top=20),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attention", "attention", "append", "w4", "w4", "logprobs", "logprobs"))
    if op == "attention":
        dtype, hd, nkv, page = rng.choice(("bf16", "bf16", "fp32")), rng.choice((32, 64, 128)), rng.choice((1, 2, 4, 8)), rng.choice((8, 16, 32, 64))
        batch = _spread(rng, 1, 200)
        most = MOST_KEY_BYTES // (batch * nkv * hd * 2 * BYTES[dtype])
        return dict(op=op, dtype=dtype, batch=batch, nq=nkv * rng.choice((1, 2, 4, 7, 8)), nkv=nkv, hd=hd, page=page,
                    longest=_spread(rng, 1, min(most, 40000)), ragged=rng.random() < 0.7)
    if op == "append":
        batch = _spread(rng, 1, 100)
        nkv = rng.choice((1, 2, 4, 8))
        return dict(op=op, source=rng.choice(("fp32", "bf16")), dtype=rng.choice(("bf16", "bf16", "fp32")), batch=batch,
                    rows=max(batch, _spread(rng, 1, 8000)), nq=nkv * rng.choice((1, 2, 4, 7)), nkv=nkv, hd=rng.choice((32, 64, 128)),
                    page=rng.choice((8, 16, 32, 64)), before=_spread(rng, 1, 4000) - 1)
    if op == "w4":
        group = rng.choice((32, 64, 128))
        K = group * max(1, _spread(rng, 256, 14336) // group)
        return dict(op=op, rows=rng.choice((1, 1, 2, 3, 4, 5, 8, 9, 13, 16, 24, 33, 64)), N=min(_spread(rng, 100, 40000), MOST_WEIGHTS // K), K=K, group=group)
    dtype, V = rng.choice(("bf16", "fp32")), _spread(rng, 500, 160000)
    return dict(op=op, dtype=dtype, rows=_spread(rng, 1, min(3000, (80 << 20) // V)), V=V, top=rng.choice((0, 1, 5, 8, 20, 32)))


def lengths(case):
    """Tokens of each sequence: all of them `longest`, or evenly spread from one to it."""
    b, n = case["batch"], case["longest"]
    return [n if not case["ragged"] or b == 1 else 1 + (n - 1) * i // (b - 1) for i in range(b)]


def counts(case):
    """New rows of each sequence, `rows` in all, at least one each and no two alike where there are enough."""
    b, n = case["batch"], case["rows"] - case["batch"]
    cut = [n * i * i // (b * b) for i in range(b + 1)]
    return [1 + cut[i + 1] - cut[i] for i in range(b)]


def starts(case):
    """Tokens of each sequence that the cache holds before the call."""
    return [case["before"] * (i + 1) // case["batch"] for i in range(case["batch"])]


def _randn(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _cache(g, case, tokens):
    """Pools [kv head, page, token in page, head dim] and a page table whose sequences have their pages in any order."""
    page, per_seq = case["page"], -(-max(tokens) // case["page"])
    n_pages = case["batch"] * per_seq
    shape = (case["nkv"], n_pages, page, case["hd"])
    table = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).view(case["batch"], per_seq)
    dtype = DTYPES[case["dtype"]]
    return dict(k_pool=_randn(g, *shape, dtype=dtype), v_pool=_randn(g, *shape, dtype=dtype), page_table=table.contiguous())


def rope_table(positions, hd, theta=10000.0):
    """Cosine and sine of every position and pair, [positions, 2, hd / 2], angles in 64 bits."""
    f = theta ** (-torch.arange(0, hd, 2, dtype=torch.float64, device="cuda") / hd)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack((a.cos(), a.sin()), dim=1).to(torch.float32).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = dict(case=case)
    if case["op"] == "attention":
        lens = _ints(lengths(case))[torch.randperm(case["batch"], generator=g, device="cuda")].contiguous()
        s.update(_cache(g, case, lengths(case)), kv_lens=lens, q=_randn(g, case["batch"], case["nq"], case["hd"], std=1.5, dtype=DTYPES[case["dtype"]]))
    elif case["op"] == "append":
        n, before = counts(case), starts(case)
        tokens = [a + b for a, b in zip(n, before)]
        edges = np.concatenate(([0], np.cumsum(n)))
        s.update(_cache(g, case, tokens), kv_lens=_ints(before), row_starts=None if case["rows"] == case["batch"] else _ints(edges.tolist()),
                 rope=rope_table(max(tokens), case["hd"]),
                 qkv=_randn(g, case["rows"], case["nq"] + 2 * case["nkv"], case["hd"], dtype=DTYPES[case["source"]]))
    elif case["op"] == "w4":
        N, K, group = case["N"], case["K"], case["group"]
        codes = (torch.randn(N, K, generator=g, device="cuda") * 2.4).round_().clamp_(-8, 7).add_(8).to(torch.uint8)
        s.update(codes=(codes[:, 0::2] | (codes[:, 1::2] << 4)).contiguous(), A=_randn(g, case["rows"], K, dtype=torch.bfloat16),
                 scales=(0.008 * (0.5 + torch.rand(N, K // group, generator=g, device="cuda"))).to(torch.bfloat16))
    else:
        s.update(logits=_randn(g, case["rows"], case["V"], std=3.0, dtype=DTYPES[case["dtype"]]),
                 tokens=torch.randint(0, case["V"], (case["rows"],), generator=g, device="cuda", dtype=torch.int32))
    return s


def run(state):
    case = state["case"]
    if own:
        return _call(state)
    if case["op"] == "attention":
        return plain_attention(state)
    if case["op"] == "append":
        return plain_append(state)
    if case["op"] == "w4":
        return plain_w4(state)
    return plain_logprobs(state)


def _call(s):
    """What a user's program calls."""
    from paper_2510_19705_b200 import binding
    op = s["case"]["op"]
    if op == "attention":
        return binding.hsd_paged_attention(s["q"], s["k_pool"], s["v_pool"], s["page_table"], s["kv_lens"])
    if op == "append":
        q = binding.hsd_kv_append(s["qkv"], s["k_pool"], s["v_pool"], s["page_table"], s["kv_lens"], s["rope"], s["row_starts"])
        return q, s["k_pool"], s["v_pool"]
    if op == "w4":
        return binding.hsd_gemm_w4(s["A"], s["codes"], s["scales"])
    return binding.hsd_token_logprobs(s["logits"], s["tokens"], s["case"]["top"])


def plain_attention(s):
    q, table, lens = s["q"].float(), s["page_table"].long(), s["kv_lens"].long()
    b, nq, hd = q.shape
    nkv, _, page, _ = s["k_pool"].shape
    n = table.shape[1] * page
    k = s["k_pool"][:, table].float().reshape(nkv, b, n, hd).transpose(0, 1)
    v = s["v_pool"][:, table].float().reshape(nkv, b, n, hd).transpose(0, 1)
    x = (q.view(b, nkv, nq // nkv, hd) @ k.transpose(2, 3)) * (hd ** -0.5)
    here = torch.arange(n, device=q.device) < lens[:, None]
    x = x.masked_fill(~here[:, None, None, :], -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    e = torch.exp(x - torch.where(top == -math.inf, torch.zeros_like(top), top))
    o = (e @ v) / e.sum(dim=-1, keepdim=True).clamp_min(1e-30)
    return o.reshape(b, nq, hd).to(s["q"].dtype)


def plain_append(s):
    qkv, table, before, rope = s["qkv"].float(), s["page_table"].long(), s["kv_lens"].long(), s["rope"]
    nkv, _, page, hd = s["k_pool"].shape
    rows, heads, _ = qkv.shape
    nq = heads - 2 * nkv
    r = torch.arange(rows, device=qkv.device)
    if s["row_starts"] is None:
        seq, at = r, before
    else:
        edges = s["row_starts"].long()
        seq = (r[:, None] >= edges[None, 1:]).sum(dim=1)
        at = before[seq] + r - edges[seq]
    x, v = qkv[:, :nq + nkv], qkv[:, nq + nkv:]
    cos, sin = rope[at, 0][:, None], rope[at, 1][:, None]
    lo, hi = x[..., :hd // 2], x[..., hd // 2:]
    y = torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), dim=-1).to(s["k_pool"].dtype)
    pages = table[seq, at // page]
    s["k_pool"][:, pages, at % page] = y[:, nq:].transpose(0, 1)
    s["v_pool"][:, pages, at % page] = v.transpose(0, 1).to(s["v_pool"].dtype)
    return y[:, :nq].contiguous(), s["k_pool"], s["v_pool"]


def plain_w4(s):
    codes, scales = s["codes"], s["scales"].float()
    N, half = codes.shape
    w = torch.stack((codes & 15, codes >> 4), dim=-1).float() - 8.0
    w = (w.view(N, scales.shape[1], -1) * scales[:, :, None]).view(N, 2 * half)
    return s["A"].float() @ w.T


def _order(x):
    """Whole numbers that sort as the stored values do, the lower token first among equals."""
    bits = (x + 0.0).contiguous().view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
    return (bits << 32) - torch.arange(x.shape[-1], device=x.device)


def plain_logprobs(s):
    x, tok, top = s["logits"].float(), s["tokens"].long()[:, None], s["case"]["top"]
    m = x.amax(dim=-1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    total = e.sum(dim=-1, keepdim=True)
    entropy = torch.log(total) - (e * d).sum(dim=-1, keepdim=True) / total
    lp = d - torch.log(total)
    key = _order(x)
    rank = (key > key.gather(1, tok)).sum(dim=1)
    ids = torch.topk(key, top, dim=1).indices
    return lp.gather(1, tok)[:, 0], entropy[:, 0], rank.to(torch.int32), ids.to(torch.int32), lp.gather(1, ids)


def work(case):
    op = case["op"]
    if op == "attention":
        keys, e = sum(lengths(case)), BYTES[case["dtype"]]
        io = case["batch"] * (2 * case["nq"] * case["hd"] * e + 4)
        return dict(bytes=keys * case["nkv"] * case["hd"] * 2 * e + io + 4 * -(-keys // case["page"]), flops=4 * keys * case["nq"] * case["hd"])
    if op == "append":
        heads, positions = case["nq"] + 2 * case["nkv"], min(case["rows"], max(a + b for a, b in zip(counts(case), starts(case))))
        return dict(bytes=case["rows"] * heads * case["hd"] * (BYTES[case["source"]] + BYTES[case["dtype"]]) + positions * case["hd"] * 4,
                    flops=case["rows"] * (case["nq"] + case["nkv"]) * case["hd"] * 3)
    if op == "w4":
        R, N, K = case["rows"], case["N"], case["K"]
        return dict(bytes=N * K // 2 + 2 * N * (K // case["group"]) + 2 * R * K + 4 * R * N, flops=2 * R * N * K)
    n = case["rows"] * case["V"]
    return dict(bytes=n * BYTES[case["dtype"]] + case["rows"] * (16 + 8 * case["top"]), flops=5 * n)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attention":
        b, nq, hd = s["q"].shape
        nkv, _, page, _ = s["k_pool"].shape
        out = torch.zeros(b, nq, hd, dtype=torch.float64, device="cuda")
        for i, n in enumerate(s["kv_lens"].tolist()):
            pages = s["page_table"][i, :-(-n // page)].long()
            for h in range(nkv):
                k, v = (s[p][h].index_select(0, pages).reshape(-1, hd)[:n].double() for p in ("k_pool", "v_pool"))
                of = slice(h * (nq // nkv), (h + 1) * (nq // nkv))
                x = torch.einsum("gd,nd->gn", s["q"][i, of].double(), k) / math.sqrt(hd)
                out[i, of] = torch.einsum("gn,nd->gd", torch.exp(x - torch.logsumexp(x, dim=1, keepdim=True)), v)
        return out
    if case["op"] == "append":
        nkv, page, hd, nq = case["nkv"], case["page"], case["hd"], case["nq"]
        k_pool, v_pool, table = s["k_pool"].double().cpu().numpy(), s["v_pool"].double().cpu().numpy(), s["page_table"].cpu().numpy()
        x, rope = s["qkv"].double().cpu().numpy(), s["rope"].double().cpu().numpy()
        q, r = np.empty((case["rows"], nq, hd)), 0
        for b, (n, before) in enumerate(zip(counts(case), starts(case))):
            for p in range(before, before + n):
                z = (x[r, :nq + nkv, :hd // 2] + 1j * x[r, :nq + nkv, hd // 2:]) * (rope[p, 0] + 1j * rope[p, 1])
                y = np.concatenate((z.real, z.imag), axis=-1)
                q[r] = y[:nq]
                k_pool[:, table[b, p // page], p % page] = y[nq:]
                v_pool[:, table[b, p // page], p % page] = x[r, nq + nkv:]
                r += 1
        return q, k_pool, v_pool
    if case["op"] == "w4":
        parts, group = [], case["group"]
        a = s["A"].double().view(case["rows"], -1, group)
        for n in range(0, case["N"], 2048):
            c = s["codes"][n:n + 2048].long()
            w = torch.empty(c.shape[0], case["K"], dtype=torch.float64, device="cuda")
            w[:, 0::2], w[:, 1::2] = (c % 16 - 8).double(), (c // 16 - 8).double()
            sums = torch.einsum("rgk,ngk->rng", a, w.view(c.shape[0], -1, group))
            parts.append((sums * s["scales"][n:n + 2048].double()).sum(dim=2))
        return torch.cat(parts, dim=1)
    x = s["logits"].double()
    lp = x - torch.logsumexp(x, dim=1, keepdim=True)
    entropy = -(lp.exp() * lp).sum(dim=1)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
    return lp.gather(1, s["tokens"].long()[:, None])[:, 0], entropy, None, None, lp.gather(1, order)
