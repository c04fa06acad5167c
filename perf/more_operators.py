"""Measured cases of the operators of a decoding step over a batch of continuations of one prompt: appending rows whose queries and
keys are normalised per head and rotated (hsd_kv_append_norm), attention over a shared prefix and each sequence's own tokens
(hsd_prefix_attention), and products in 8-bit integers with scales of tokens and channels (hsd_gemm_w8).

`own` chooses what run() does: the plain forms in elementary torch operations, or the calls of the package."""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"fp32": 4, "bf16": 2}
MOST_SCORES = 100 * 32 * 40300    # rows x query heads x keys of a drawn attention: the largest listed one's
MOST_PRODUCT = 4096 * 14336 * 4096
MOST_WEIGHTS = 28672 * 4096
EPS = 1e-6


def listed():
    return [
        # four continuations of the 8B shape's prompt of 1024 tokens, a few tokens in: latency
        dict(name="prefix, 4 x 1024", op="prefix", dtype="bf16", batch=4, most=1, nq=32, nkv=8, hd=128, page=16, prefix=1024, own=40),
        # samples of one long prompt, hundreds of tokens each
        dict(name="prefix, 64 x 8192", op="prefix", dtype="bf16", batch=64, most=1, nq=32, nkv=8, hd=128, page=16, prefix=8192, own=500),
        # up to nine rows a sequence (eight drafts and one more) behind a prompt that ends inside a page
        dict(name="prefix, 16 x 9 rows, 16395", op="prefix", dtype="bf16", batch=16, most=9, nq=32, nkv=8, hd=128, page=16, prefix=16395, own=300),
        # a hundred samples of a whole document
        dict(name="prefix, 100 x 40000", op="prefix", dtype="bf16", batch=100, most=1, nq=32, nkv=8, hd=128, page=32, prefix=40000, own=300),
        # a small fp32 model's heads
        dict(name="prefix, fp32 heads of 32", op="prefix", dtype="fp32", batch=12, most=3, nq=8, nkv=2, hd=32, page=16, prefix=700, own=100),
        # a token of each of eight sequences: the projections' fp32 rows into a bf16 cache
        dict(name="append, 8 x 1", op="append", source="fp32", dtype="bf16", batch=8, rows=8, nq=32, nkv=8, hd=128, page=16, before=1024),
        # prompts of a batch, ragged, together
        dict(name="append, prompts of 7", op="append", source="bf16", dtype="bf16", batch=7, rows=8191, nq=32, nkv=8, hd=128, page=16, before=300),
        # one token through q, k and v of the 8B shape
        dict(name="w8, 1 x 6144 x 4096", op="w8", source="bf16", out="fp32", rows=1, N=6144, K=4096),
        # sixteen sequences through its gate and up
        dict(name="w8, 16 x 28672 x 4096", op="w8", source="bf16", out="fp32", rows=16, N=28672, K=4096),
        # drafts of a batch through the 1B shape's down projection, from fp32 rows
        dict(name="w8, 144 x 2048 x 5632", op="w8", source="fp32", out="fp32", rows=144, N=2048, K=5632),
        # a prompt through the 8B shape's gate, an odd number of tokens
        dict(name="w8, 4095 x 14336 x 4096", op="w8", source="bf16", out="bf16", rows=4095, N=14336, K=4096),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("prefix", "prefix", "append", "w8", "w8"))
    if op == "prefix":
        dtype, hd, nkv = rng.choice(("bf16", "bf16", "bf16", "fp32")), rng.choice((32, 64, 128, 128)), rng.choice((1, 2, 4, 8))
        nq, batch, most = nkv * rng.choice((1, 2, 4, 7, 8)), _spread(rng, 1, 200), rng.choice((1, 1, 1, 2, 4, 9))
        keys = min(MOST_SCORES // (4 if dtype == "fp32" else 1) // (batch * most * nq), 40000)
        own_keys = _spread(rng, most, max(most, min(1000, keys // 2, (1 << 28) // (batch * most * nkv * hd))))
        return dict(op=op, dtype=dtype, batch=batch, most=most, nq=nq, nkv=nkv, hd=hd, page=rng.choice((8, 16, 32, 64)), prefix=_spread(rng, 1, max(1, keys - own_keys)), own=own_keys)
    if op == "append":
        batch, nkv = _spread(rng, 1, 100), rng.choice((1, 2, 4, 8))
        return dict(op=op, source=rng.choice(("fp32", "bf16")), dtype=rng.choice(("bf16", "bf16", "fp32")), batch=batch,
                    rows=max(batch, _spread(rng, 1, 8000)), nq=nkv * rng.choice((1, 2, 4, 7)), nkv=nkv, hd=rng.choice((32, 64, 128)),
                    page=rng.choice((8, 16, 32, 64)), before=_spread(rng, 1, 4000) - 1)
    rows, K = _spread(rng, 1, 4095), 16 * _spread(rng, 16, 900)
    return dict(op=op, source=rng.choice(("bf16", "bf16", "fp32")), out=rng.choice(("fp32", "bf16")), rows=rows,
                N=max(1, min(_spread(rng, 100, 30000), MOST_WEIGHTS // K, MOST_PRODUCT // (rows * K))), K=K)


def counts(case):
    """New rows of each sequence: of an attention from one to `most`, of an append `rows` in all, at least one each."""
    b = case["batch"]
    if case["op"] == "prefix":
        return [1 + i % case["most"] for i in range(b)]
    n = case["rows"] - b
    cut = [n * i * i // (b * b) for i in range(b + 1)]
    return [1 + cut[i + 1] - cut[i] for i in range(b)]


def lengths(case):
    """Tokens of each sequence: for an attention with the prefix and the new rows, its own evenly spread; before an append."""
    b = case["batch"]
    if case["op"] == "prefix":
        return [case["prefix"] + max(n, case["own"] * (i + 1) // b) for i, n in enumerate(counts(case))]
    return [case["before"] * (i + 1) // b for i in range(b)]


def _edges(n):
    out = [0]
    for x in n:
        out.append(out[-1] + x)
    return out


def _randn(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32) * std).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def rope_table(positions, hd, theta=10000.0):
    """Cosine and sine of every position and pair, [positions, 2, hd / 2], angles in 64 bits."""
    f = theta ** (-torch.arange(0, hd, 2, dtype=torch.float64, device="cuda") / hd)
    a = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * f
    return torch.stack((a.cos(), a.sin()), dim=1).to(torch.float32).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    s = dict(case=case)
    if case["op"] == "w8":
        # weights and their scales as a program has them after packing: codes of a normal weight, a scale a channel
        R, N, K = case["rows"], case["N"], case["K"]
        s.update(codes=torch.empty(N, K, dtype=torch.int8, device="cuda"), scales=(0.02 * (0.5 + torch.rand(N, generator=g, device="cuda"))) / 127)
        for n in range(0, N, 4096):
            s["codes"][n:n + 4096] = _randn(g, min(4096, N - n), K, std=34.0).round_().clamp_(-127, 127).to(torch.int8)
        # activations with a few large channels, as behind a norm
        s["A"] = (_randn(g, R, K) * (1 + 5 * (torch.rand(K, generator=g, device="cuda") > 0.99))).to(DTYPES[case["source"]])
        return s
    n, lens, page, dtype = counts(case), lengths(case), case["page"], DTYPES[case["dtype"]]
    shared = case["prefix"] // page if case["op"] == "prefix" else 0         # whole pages that all sequences have
    most = max(lens) if case["op"] == "prefix" else max(a + b for a, b in zip(lens, n))
    of_its_own = -(-most // page) - shared
    total = shared + case["batch"] * of_its_own + 1
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.cat((order[None, :shared].expand(case["batch"], -1), order[shared:-1].view(case["batch"], of_its_own)), dim=1)
    shape = (case["nkv"], total, page, case["hd"])
    s.update(k_pool=_randn(g, *shape, dtype=dtype), v_pool=_randn(g, *shape, dtype=dtype), page_table=table.contiguous(), kv_lens=_ints(lens))
    starts = None if max(n) == 1 else _ints(_edges(n))
    if case["op"] == "prefix":
        # the prefix's last page may be a partial one of which every sequence has a copy: the list names it by itself
        pages = -(-case["prefix"] // page)
        prefix_pages = torch.cat((order[:shared], order[-1:]))[:pages].contiguous()
        s.update(q=_randn(g, sum(n), case["nq"], case["hd"], std=1.5, dtype=dtype), prefix_pages=prefix_pages, prefix_len=_ints([case["prefix"]]), row_starts=starts)
    else:
        gain = 1 + 0.3 * torch.randn(2, case["hd"], generator=g, device="cuda")
        s.update(qkv=_randn(g, case["rows"], case["nq"] + 2 * case["nkv"], case["hd"], std=2.0, dtype=DTYPES[case["source"]]), row_starts=starts,
                 rope=rope_table(most, case["hd"]), q_gain=gain[0].to(torch.bfloat16), k_gain=gain[1].to(torch.bfloat16))
    return s


def run(state):
    op = state["case"]["op"]
    if own:
        return _call(state)
    return plain_prefix(state) if op == "prefix" else plain_append(state) if op == "append" else plain_w8(state)


def _call(s):
    """What a user's program calls."""
    from paper_2510_19705_b200 import binding
    op = s["case"]["op"]
    if op == "prefix":
        return binding.hsd_prefix_attention(s["q"], s["k_pool"], s["v_pool"], s["page_table"], s["kv_lens"], s["prefix_pages"], s["prefix_len"], s["row_starts"])
    if op == "append":
        q = binding.hsd_kv_append_norm(s["qkv"], s["q_gain"], s["k_gain"], EPS, s["k_pool"], s["v_pool"], s["page_table"], s["kv_lens"], s["rope"], s["row_starts"])
        return q, s["k_pool"], s["v_pool"]
    return binding.hsd_gemm_w8(s["A"], s["codes"], s["scales"], DTYPES[s["case"]["out"]])


def _rows(s, rows):
    """Sequence of each row, its place among the sequence's new rows, and their number."""
    r = torch.arange(rows, device="cuda")
    if s["row_starts"] is None:
        return r, torch.zeros_like(r), torch.ones_like(r)
    edges = s["row_starts"].long()
    seq = (r[:, None] >= edges[None, 1:]).sum(dim=1)
    return seq, r - edges[seq], (edges[1:] - edges[:-1])[seq]


def plain_prefix(s):
    q, table, lens, P = s["q"].float(), s["page_table"].long(), s["kv_lens"].long(), s["case"]["prefix"]
    rows, nq, hd = q.shape
    nkv, _, page, _ = s["k_pool"].shape
    seq, at, new = _rows(s, rows)
    limit = lens[seq] - new + 1 + at
    front = P // page                            # sequences' own tokens begin inside of this page
    own_pages, here = table[:, front:], s["prefix_pages"].long()
    m = own_pages.shape[1] * page
    k0, v0 = (s[p][:, here].reshape(nkv, -1, hd)[:, :P].float() for p in ("k_pool", "v_pool"))
    k1, v1 = (s[p][:, own_pages].reshape(nkv, -1, m, hd)[:, seq].float() for p in ("k_pool", "v_pool"))
    x = q.view(rows, nkv, nq // nkv, hd).transpose(0, 1)                                     # [nkv, rows, group, hd]
    x0 = (x.reshape(nkv, -1, hd) @ k0.transpose(1, 2)).view(nkv, rows, -1, P)
    x1 = x @ k1.transpose(2, 3)
    pos = torch.cat((torch.arange(P, device="cuda"), front * page + torch.arange(m, device="cuda")))
    own_key = torch.arange(P + m, device="cuda") >= P
    seen = (pos < limit[:, None]) & (~own_key | (pos >= P))
    x = torch.cat((x0, x1), dim=3).mul_(hd ** -0.5).masked_fill_(~seen[None, :, None, :], -math.inf)
    top = x.amax(dim=3, keepdim=True)
    e = x.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    o = (e[..., :P].reshape(nkv, -1, P) @ v0).view(nkv, rows, -1, hd) + e[..., P:] @ v1
    o = o / e.sum(dim=3, keepdim=True).clamp_min(1e-30)
    return o.transpose(0, 1).reshape(rows, nq, hd).to(s["q"].dtype)


def plain_append(s):
    qkv, table, before, rope = s["qkv"].float(), s["page_table"].long(), s["kv_lens"].long(), s["rope"]
    nkv, _, page, hd = s["k_pool"].shape
    rows, heads, _ = qkv.shape
    nq = heads - 2 * nkv
    seq, at, _ = _rows(s, rows)
    at = before[seq] + at
    x, v = qkv[:, :nq + nkv], qkv[:, nq + nkv:]
    gain = torch.cat((s["q_gain"].float().expand(nq, hd), s["k_gain"].float().expand(nkv, hd)))
    x = x / torch.sqrt((x * x).mean(dim=2, keepdim=True) + EPS) * gain
    cos, sin = rope[at, 0][:, None], rope[at, 1][:, None]
    lo, hi = x[..., :hd // 2], x[..., hd // 2:]
    y = torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), dim=-1).to(s["k_pool"].dtype)
    pages = table[seq, at // page]
    s["k_pool"][:, pages, at % page] = y[:, nq:].transpose(0, 1)
    s["v_pool"][:, pages, at % page] = v.transpose(0, 1).to(s["v_pool"].dtype)
    return y[:, :nq].contiguous(), s["k_pool"], s["v_pool"]


def plain_w8(s):
    x = s["A"].float()
    top = x.abs().amax(dim=1, keepdim=True)
    scale = top / torch.full_like(top, 127.0)                                # (a quotient: by a number it would be a product)
    # 64 bits: a quotient next to the middle of two codes
    a = torch.round(x.double() / torch.where(scale > 0, scale, torch.ones_like(scale)).double()).clamp_(-127, 127).float()
    return ((a @ s["codes"].float().T) * scale * s["scales"]).to(DTYPES[s["case"]["out"]])


def work(case):
    op = case["op"]
    if op == "w8":
        R, N, K = case["rows"], case["N"], case["K"]
        return dict(bytes=N * K + 4 * N + R * K * BYTES[case["source"]] + R * N * BYTES[case["out"]], flops=2 * R * N * K)
    n, lens, e, hd = counts(case), lengths(case), BYTES[case["dtype"]], case["hd"]
    if op == "prefix":
        keys = case["prefix"] + sum(x - case["prefix"] for x in lens)
        seen = sum(x * (length + 1) - x * (x + 1) // 2 for x, length in zip(n, lens))
        return dict(bytes=keys * case["nkv"] * hd * 2 * e + 2 * sum(n) * case["nq"] * hd * e + 4 * -(-keys // case["page"]), flops=4 * seen * case["nq"] * hd)
    heads, positions = case["nq"] + 2 * case["nkv"], min(case["rows"], max(a + b for a, b in zip(n, lens)))
    return dict(bytes=case["rows"] * heads * hd * (BYTES[case["source"]] + e) + positions * hd * 4, flops=case["rows"] * (case["nq"] + case["nkv"]) * hd * 7)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "w8":
        x, out = s["A"].double(), []
        scale = (x.abs().amax(dim=1) / 127).float().double()                 # the scale is a number of 32 bits by definition
        a = torch.where(scale[:, None] > 0, x / scale[:, None], torch.zeros_like(x)).round().clamp(-127, 127)
        for n in range(0, case["N"], 4096):                                  # whole numbers below 2^53: exact
            out.append(torch.einsum("rk,nk->rn", a, s["codes"][n:n + 4096].double()) * torch.outer(scale, s["scales"][n:n + 4096].double()))
        return torch.cat(out, dim=1)
    n, lens, page, hd, nq, nkv = counts(case), lengths(case), case["page"], case["hd"], case["nq"], case["nkv"]
    if case["op"] == "prefix":
        P, group, edges = case["prefix"], nq // nkv, _edges(n)
        out = torch.empty(edges[-1], nq, hd, dtype=torch.float64, device="cuda")
        pos = torch.arange(max(lens), device="cuda")
        for h in range(nkv):
            of = slice(h * group, (h + 1) * group)
            front = s["prefix_pages"].long()[pos[:P] // page], pos[:P] % page
            k0, v0 = (s[p][h][front].double() for p in ("k_pool", "v_pool"))
            for b, length in enumerate(lens):
                behind = s["page_table"][b].long()[pos[P:length] // page], pos[P:length] % page
                k, v = (torch.cat((x, s[p][h][behind].double())) for x, p in ((k0, "k_pool"), (v0, "v_pool")))
                x = torch.einsum("rgd,nd->rgn", s["q"][edges[b]:edges[b + 1], of].double(), k) / math.sqrt(hd)
                last = length - n[b] + torch.arange(n[b], device="cuda")
                x = torch.where(pos[:length] <= last[:, None, None], x, -math.inf)
                out[edges[b]:edges[b + 1], of] = torch.einsum("rgn,nd->rgd", torch.softmax(x, dim=2), v)
        return out
    k_pool, v_pool, rope, r0 = s["k_pool"].double(), s["v_pool"].double(), s["rope"].double(), 0
    x, q = s["qkv"].double(), []
    for b, (rows, before) in enumerate(zip(n, lens)):
        pos = torch.arange(before, before + rows, device="cuda")
        where = s["page_table"][b].long()[pos // page], pos % page
        z = x[r0:r0 + rows, :nq + nkv]
        z = z * torch.rsqrt(z.square().mean(dim=2, keepdim=True) + EPS)
        z[:, :nq] *= s["q_gain"].double()
        z[:, nq:] *= s["k_gain"].double()
        z = torch.complex(z[..., :hd // 2], z[..., hd // 2:]) * torch.complex(rope[pos, 0], rope[pos, 1])[:, None]
        y = torch.cat((z.real, z.imag), dim=2)
        q.append(y[:, :nq])
        k_pool[(slice(None),) + where], v_pool[(slice(None),) + where] = y[:, nq:].transpose(0, 1), x[r0:r0 + rows, nq + nkv:].transpose(0, 1)
        r0 += rows
    return torch.cat(q), k_pool, v_pool
