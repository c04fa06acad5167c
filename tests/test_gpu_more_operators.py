"""The operators of a decoding step over continuations of one prompt against plain implementations in 64 bits: appends with norms by head,
products in 8-bit integers, attention over a shared prefix.

Tolerances count roundings: half a step of the output's type, 2^-24 for each fp32 operation, 2^-23 where the tensor cores' adders may
cut off instead of rounding."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
BF16, FP32 = torch.bfloat16, torch.float32


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape, dtype=FP32, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def cache(g, batch, nkv, hd, page, per_seq, dtype, order="head", spare=3):
    """Pools in the engine's order or token-major, a page table in any order, pages that no sequence has."""
    n = batch * per_seq + spare
    pools = []
    for _ in range(2):
        if order == "head":
            pools.append(randn(g, nkv, n, page, hd, dtype=dtype))
        else:
            pools.append(randn(g, n, page, nkv, hd, dtype=dtype).permute(2, 0, 1, 3))
    table = torch.randperm(n, generator=g, device="cuda")[:batch * per_seq].view(batch, per_seq).to(torch.int32).contiguous()
    return pools[0], pools[1], table


# ------------------------------------------------------------------------------------------------ append with norms
def append64(qkv, gains, eps, table, before, rope, starts, nkv, pool_shape):
    """Rows' (page, token, queries, keys, values, sizes of the rotation's terms) in 64 bits; rows that are skipped are missing."""
    rows, heads, hd = qkv.shape
    nq, (n_pages, page) = heads - 2 * nkv, pool_shape
    x, t, table = qkv.double().cpu(), rope.double().cpu(), table.cpu()
    gain = torch.ones(nq + nkv, hd, dtype=torch.float64)
    for g, at in zip(gains, (slice(0, nq), slice(nq, None))):
        if g is not None:
            gain[at] = g.double().cpu()
    found = {}
    for b, len0 in enumerate(before):
        for r in range(starts[b], min(starts[b + 1], rows)):
            p = len0 + r - starts[b]
            if len0 < 0 or p >= t.shape[0] or p >= table.shape[1] * page or not 0 <= int(table[b, p // page]) < n_pages:
                continue
            z = x[r, :nq + nkv]
            z = z / torch.sqrt(z.square().mean(dim=1, keepdim=True) + eps) * gain
            lo, hi = z[:, :hd // 2], z[:, hd // 2:]
            y = torch.cat((lo * t[p, 0] - hi * t[p, 1], hi * t[p, 0] + lo * t[p, 1]), dim=1)
            size = torch.cat(((lo * t[p, 0]).abs() + (hi * t[p, 1]).abs(), (hi * t[p, 0]).abs() + (lo * t[p, 1]).abs()), dim=1)
            found[r] = (int(table[b, p // page]), p % page, y[:nq], y[nq:], x[r, nq + nkv:], size)
    return found


def check_append(lib, qkv, gains, eps, k, v, table, before, rope, starts=None):
    nkv, n_pages, page, hd = k.shape
    q_out = torch.full((qkv.shape[0], qkv.shape[1] - 2 * nkv, hd), 7.0, dtype=k.dtype, device="cuda")
    k0, v0 = k.clone(), v.clone()
    edges = list(range(len(before) + 1)) if starts is None else starts
    found = append64(qkv, gains, eps, table, before, rope, edges, nkv, (n_pages, page))
    assert lib.hsd_kv_append_norm(qkv, *gains, eps, k, v, table, ints(before), rope, None if starts is None else ints(starts), q_out) is q_out
    touched = torch.zeros(n_pages, page, dtype=torch.bool)
    step = HALF_STEP[k.dtype]
    kc, vc, qc = k.cpu(), v.cpu(), q_out.cpu()
    for r, (pg, t, qy, ky, vx, size) in found.items():
        touched[pg, t] = True
        for out, want, s in ((qc[r], qy, size[:qy.shape[0]]), (kc[:, pg, t], ky, size[qy.shape[0]:])):
            # the mean: a chain of 16 and three sums, halved by the root; root, two products, the rotation's three operations
            assert bool(((out.double() - want).abs() <= step * want.abs() + 18 * 2.0 ** -24 * s + 1e-37).all())
        assert torch.equal(vc[:, pg, t], vx.to(FP32).to(k.dtype))
    left = torch.tensor([r for r in range(qkv.shape[0]) if r not in found], dtype=torch.long, device="cuda")
    assert bool((q_out[left] == 7.0).all())                                  # skipped rows: as they were
    keep = ~touched.cuda()
    assert torch.equal(k[:, keep], k0[:, keep]) and torch.equal(v[:, keep], v0[:, keep])
    k.copy_(k0), v.copy_(v0)
    zeros = lib.hsd_kv_append_norm(qkv, *gains, eps, k, v, table, ints(before), rope, None if starts is None else ints(starts))
    assert bool((zeros[left] == 0).all()) and torch.equal(zeros[sorted(found)], q_out[sorted(found)])
    return found


@pytest.mark.parametrize("source", [BF16, FP32])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("hd,nq,nkv,page,order", [(32, 5, 2, 16, "head"), (64, 1, 1, 3, "token"), (128, 8, 2, 16, "token"), (64, 0, 3, 8, "head"), (128, 1, 1, 16, "head")])
def test_append_norm_one_token_each(lib, source, dtype, hd, nq, nkv, page, order):
    g = gen(hd + nq)
    before = [0, 1, 15, 16, 31, -1, 40]
    k, v, table = cache(g, 7, nkv, hd, page, -(-41 // page), dtype, order)
    gains = [1 + randn(g, hd, std=0.3).to(source) for _ in range(2)]
    found = check_append(lib, randn(g, 7, nq + 2 * nkv, hd, dtype=source, std=3.0), gains, 1e-6, k, v, table, before, lib.rope_table(64, hd))
    assert sorted(found) == [0, 1, 2, 3, 4, 6]


@pytest.mark.parametrize("gains", [(None, None), (FP32, None), (None, BF16)])
@pytest.mark.parametrize("eps", [0.0, 1e-5, 10.0])
def test_append_norm_without_gains_and_other_eps(lib, gains, eps):
    g = gen(2)
    k, v, table = cache(g, 3, 2, 64, 16, 2, FP32)
    gains = [None if t is None else randn(g, 64, dtype=t) for t in gains]
    check_append(lib, randn(g, 3, 7, 64, std=1e-3), gains, eps, k, v, table, [3, 0, 31], lib.rope_table(64, 64))


@pytest.mark.parametrize("rows", [1, 40, 301, 701, 2503])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_append_norm_ragged_rows(lib, rows, dtype):
    g = gen(rows)
    batch = 70
    cut = sorted(torch.randint(0, rows + 1, (batch - 1,), generator=torch.Generator().manual_seed(rows)).tolist())
    starts = [0] + cut + [rows]
    before = [(i * 37) % 50 for i in range(batch)]
    longest = max(b + starts[i + 1] - starts[i] for i, b in enumerate(before))
    k, v, table = cache(g, batch, 1, 32, 16, -(-longest // 16), dtype)
    gains = [randn(g, 32), randn(g, 32)]
    assert len(check_append(lib, randn(g, rows, 4, 32), gains, 1e-6, k, v, table, before, lib.rope_table(longest, 32), starts)) == rows


def test_append_norm_skips_what_has_no_place_and_takes_rows_that_lie_apart(lib):
    g = gen(3)
    k, v, table = cache(g, 4, 1, 64, 16, 2, BF16)
    table[1, 1], table[2, 0] = -1, k.shape[1]
    qkv = randn(g, 30, 5 * 64)[:, 64:256].unflatten(1, (3, 64))
    found = check_append(lib, qkv, [randn(g, 64), None], 1e-6, k, v, table, [28, 14, 0, 18], lib.rope_table(30, 64), [2, 8, 13, 16, 25])
    assert sorted(found) == [2, 3, 8, 9] + list(range(16, 25))


def test_append_norm_of_zeros_and_of_values_that_are_not_finite(lib):
    g = gen(4)
    k, v, table = cache(g, 1, 2, 64, 16, 1, FP32)
    qkv = randn(g, 1, 6, 64)
    qkv[0, 0], qkv[0, 1, 3], qkv[0, 4, 5] = 0, float("nan"), float("inf")
    q = lib.hsd_kv_append_norm(qkv, None, None, 1e-6, k, v, table, ints([0]), lib.rope_table(4, 64))
    at = int(table[0, 0])
    assert bool((q[0, 0] == 0).all()) and bool(q[0, 1].isnan().all())
    assert bool(k[:, at, 0].isfinite().all()) and torch.equal(v[:, at, 0], qkv[0, 4:])


# ------------------------------------------------------------------------------------------------ 8-bit products
def quantize64(x):
    """(codes as doubles, scales): the nearest whole numbers of scales of 32 bits."""
    x = x.double()
    bad = ~x.isfinite().all(dim=1)
    scale = (x.abs().amax(dim=1) / 127).float()
    c = torch.round(x / torch.where(scale > 0, scale, torch.ones_like(scale)).double()[:, None]).clamp(-127, 127)
    c[bad] = 0
    scale[bad] = float("nan")
    return c, scale


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,K", [(1, 1), (3, 7), (5, 16), (2, 255), (7, 4096), (300, 1000), (2, 16384), (3, 16392), (1, 50001), (4095, 64)])
def test_quantized_rows(lib, dtype, rows, K):
    g = gen(K + rows)
    x = randn(g, rows, K, dtype=dtype, std=2.0)
    codes, scales = lib.hsd_quantize_rows(x)
    assert codes.dtype == torch.int8 and codes.shape == (rows, K) and scales.dtype == FP32 and scales.shape == (rows,)
    c, s = quantize64(x)
    assert torch.equal(scales, s) and torch.equal(codes.double(), c)


def test_quantized_rows_between_two_codes(lib):
    """Values at and next to the middle of two codes, where a quotient's own rounding would decide."""
    g = gen(1)
    scale = torch.rand(64, 1, generator=g, device="cuda") * 10.0 ** torch.randint(-30, 30, (64, 1), generator=g, device="cuda").float()
    half = torch.arange(-126, 126, device="cuda") + 0.5
    x = (half * scale.double()).float()
    x = torch.cat((x, torch.nextafter(x, torch.zeros_like(x)), torch.nextafter(x, 1e38 * torch.ones_like(x)), 127 * scale), dim=1)
    codes, scales = lib.hsd_quantize_rows(x)
    c, s = quantize64(x)
    assert torch.equal(scales, s) and torch.equal(codes.double(), c)
    y = half.repeat(3, 1).contiguous()
    y[:, 0] = 127                                                            # scale 1: exact middles go to the even code
    assert torch.equal(lib.hsd_quantize_rows(y)[0].double(), y.double().round())


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_quantized_rows_of_zeros_small_and_large_values_and_what_is_not_finite(lib, dtype):
    x = randn(gen(2), 9, 64, dtype=dtype)
    x[0] = 0
    x[1, 5], x[2, 6], x[3, 7] = float("inf"), float("nan"), -float("inf")
    x[4] *= torch.finfo(dtype).tiny                                          # subnormal scales
    x[5] = torch.finfo(dtype).max * torch.where(x[5] > 0, 1.0, -1.0).to(dtype)
    x[6] = 0
    x[6, 3] = torch.finfo(dtype).smallest_normal / 64                        # the scale is 0 or the smallest number
    x[7] *= 1e-33
    codes, scales = lib.hsd_quantize_rows(x)
    c, s = quantize64(x)
    assert torch.equal(scales.nan_to_num(-1), s.nan_to_num(-1)) and torch.equal(codes.double(), c)


def test_quantized_rows_that_lie_apart(lib):
    x = randn(gen(3), 11, 200, dtype=BF16)
    for part in (x[:, 8:136], x[:, 3:135], x[::2], x[:1, 1:70]):
        codes, scales = lib.hsd_quantize_rows(part)
        c, s = quantize64(part)
        assert torch.equal(scales, s) and torch.equal(codes.double(), c)


def check_w8(lib, A, codes, scales, out_dtype=FP32, **more):
    got = lib.hsd_gemm_w8(A, codes, scales, out_dtype, **more)
    c, s = (A, more["a_scales"]) if A.dtype == torch.int8 else quantize64(A)
    want = torch.cat([(c.double() @ codes[n:n + 8192].double().T) for n in range(0, codes.shape[0], 8192)], dim=1) * torch.outer(s.double(), scales.double())
    assert got.dtype == out_dtype and got.shape == want.shape
    # the whole number's rounding, two products, the output's own
    off, bound = (got.double() - want).abs(), (3.01 * 2.0 ** -24 + (2.0 ** -8 if out_dtype == BF16 else 0)) * want.abs() + 1e-37
    assert bool((off <= bound).all()), (float((off / bound).max()), int((off > bound).sum()))
    return got


def weights(g, N, K):
    return torch.randint(-128, 128, (N, K), generator=g, device="cuda", dtype=torch.int8), 0.01 * (0.1 + torch.rand(N, generator=g, device="cuda"))


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 32, 33, 64, 65, 128, 129, 255, 256, 257, 300, 513])
@pytest.mark.parametrize("N,K", [(1, 16), (17, 144), (100, 4096), (1001, 2064)])
def test_w8_products(lib, rows, N, K):
    g = gen(N + rows)
    codes, scales = weights(g, N, K)
    check_w8(lib, randn(g, rows, K, dtype=BF16), codes, scales)
    check_w8(lib, randn(g, rows, K), codes, scales, BF16)


@pytest.mark.parametrize("rows,N,K,out", [(1, 4096, 4096, FP32), (1, 6144, 4096, BF16), (16, 28672, 4096, FP32), (200, 2048, 5632, BF16), (144, 32000, 2048, FP32),
                                          (40, 300, 14336, FP32), (700, 6144, 4096, BF16), (2049, 4096, 1024, FP32), (3, 9473, 512, FP32)])
def test_w8_products_of_layers(lib, rows, N, K, out):
    g = gen(N)
    A, (codes, scales) = randn(g, rows, K, dtype=BF16), weights(g, N, K)
    got = check_w8(lib, A, codes, scales, out)
    into = torch.empty(rows, N, dtype=out, device="cuda")
    assert lib.hsd_gemm_w8(A, codes, scales, out, out=into) is into and torch.equal(into, got)
    a, s = lib.hsd_quantize_rows(A)
    assert torch.equal(check_w8(lib, a, codes, scales, out, a_scales=s), got)


@pytest.mark.parametrize("rows", [5, 300])
def test_w8_sums_are_exact_at_their_largest(lib, rows):
    K = (1 << 17) - 16
    A, w = torch.full((rows, K), -128, dtype=torch.int8, device="cuda"), torch.full((200, K), -128, dtype=torch.int8, device="cuda")
    w[::2], w[7], w[7, 5] = 127, 0, 1
    got = lib.hsd_gemm_w8(A, w, torch.ones(200, device="cuda"), a_scales=torch.ones(rows, device="cuda"))
    want = torch.full((200,), 16384.0 * K, dtype=torch.float64)
    want[::2], want[7] = -128.0 * 127 * K, -128
    assert torch.equal(got.cpu(), want.float().expand(rows, 200))


@pytest.mark.parametrize("rows", [3, 400])
def test_w8_keeps_what_is_not_finite_to_its_row(lib, rows):
    g = gen(5)
    A, (codes, scales) = randn(g, rows, 256, dtype=BF16), weights(g, 300, 256)
    want = lib.hsd_gemm_w8(A, codes, scales)
    A2, s2 = A.clone(), scales.clone()
    A2[1, 7], s2[5] = float("nan"), float("inf")
    A2[2] = 0
    got = lib.hsd_gemm_w8(A2, codes, s2)
    other, cols = [r for r in range(rows) if r not in (1, 2)], [i for i in range(300) if i != 5]
    assert bool(got[1].isnan().all()) and not bool(got[other][:, 5].isfinite().any()) and bool((got[2][cols] == 0).all())
    assert torch.equal(got[other][:, cols], want[other][:, cols])


def test_w8_packed_weights_near_the_bf16_product(lib):
    g = gen(6)
    W, A = randn(g, 200, 512, dtype=BF16, std=0.02), randn(g, 40, 512, dtype=BF16)
    codes, scales = lib.hsd_quantize_rows(W)
    got = check_w8(lib, A, codes, scales)
    c, s = quantize64(A)
    # a weight is off by half of its row's scale at most, and an activation too
    a = (c * s.double()[:, None]).abs()
    bound = 0.5001 * (a.sum(dim=1)[:, None] * scales.double() + s.double()[:, None] * W.double().abs().sum(dim=1))
    assert bool(((got.double() - A.double() @ W.double().T).abs() <= bound).all())


def test_w8_captured_on_other_streams_and_two_at_once(lib):
    g = gen(7)
    codes, scales = weights(g, 3000, 1024)
    xs = [randn(g, n, 1024, dtype=BF16) for n in (9, 300)]
    want = [lib.hsd_gemm_w8(x, codes, scales) for x in xs]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x in xs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(lib.hsd_gemm_w8(x, codes, scales))
        graphs.append(graph)
    fresh = [randn(g, *x.shape, dtype=BF16) for x in xs]
    for new in (xs, fresh):
        keep = [x.clone() for x in new]
        for x, y in zip(xs, keep):
            x.copy_(y)
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for x, out in zip(xs, outs):
            assert torch.equal(out, lib.hsd_gemm_w8(x, codes, scales))
    assert not torch.equal(outs[0], want[0])
    want = [lib.hsd_gemm_w8(x, codes, scales) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[] for _ in xs]
    for _ in range(20):
        for i, (x, st) in enumerate(zip(xs, streams)):
            with torch.cuda.stream(st):
                got[i].append(lib.hsd_gemm_w8(x, codes, scales))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])


# ------------------------------------------------------------------------------------------------ attention over a shared prefix
def counts_of(starts, batch):
    return [(b, b + 1) for b in range(batch)] if starts is None else list(zip(starts[:-1], starts[1:]))


def prefix64(q, k_pool, v_pool, table, lens, pages, P, starts, scale):
    """(out, sum of weights times |v|, the largest sum of |q||k|), all in 64 bits; rows without a sequence are NaN."""
    rows, nq, hd = q.shape
    nkv, n_pages, page, _ = k_pool.shape
    out, size, most = (torch.full((rows, nq, n), float("nan"), dtype=torch.float64) for n in (hd, hd, 1))
    P = min(max(P, 0), len(pages) * page)
    room = table.shape[1] * page
    kc, vc, qc = k_pool.double().cpu(), v_pool.double().cpu(), q.double().cpu()
    for b, (r0, r1) in enumerate(counts_of(starts, len(lens))):
        n = min(max(lens[b], 0), max(room, P))
        where = [(int(pages[p // page]) if p < P else int(table[b, p // page]) if p < room else -1, p % page, p) for p in range(n)]
        where = [x for x in where if 0 <= x[0] < n_pages]
        for r in range(r0, min(r1, rows)):
            limit = n - (r1 - r0) + 1 + r - r0
            seen = [x for x in where if x[2] < limit]
            out[r], size[r], most[r] = 0, 0, 0
            if not seen or n - (r1 - r0) + 1 < P:                            # without the whole prefix: zeros
                continue
            a, t, _ = (torch.tensor(x) for x in zip(*seen))
            for h in range(nq):
                k, v, x = kc[h * nkv // nq][a, t], vc[h * nkv // nq][a, t], qc[r, h]
                w = torch.softmax(k @ x * scale, dim=0)
                out[r, h], size[r, h], most[r, h] = w @ v, w @ v.abs(), (k.abs() @ x.abs()).max() * abs(scale)
    return out, size, most


def check_prefix(lib, q, k, v, table, lens, pages, P, starts=None, scale=None, long=True):
    """With the list of pages as it is and, for bf16 (`long`), with more of them behind the prefix's end: a call whose list has room for many
    keys takes the tensor-memory kernel."""
    rows, nq, hd = q.shape
    nkv, page = k.shape[0], k.shape[2]
    want, size, most = prefix64(q, k, v, table.cpu(), lens, pages.cpu(), P, starts, hd ** -0.5 if scale is None else scale)
    none = want[:, 0, 0].isnan()
    # as in the attention by sequence: a score's sum and its exponential; tiles added one after the other; bf16 weights of 16 bits, and
    # chains of up to 2048 keys in the tensor cores' adders, two products for every 16 keys
    weight = (hd + 4) * 2.0 ** -23 * most + 2.0 ** -21 + (max(max(lens), P) / 8 + 64) * 2.0 ** -24 + (2.0 ** -16 if q.dtype == BF16 else 0)
    chain = 256 * 2.0 ** -23 if q.dtype == BF16 else 0
    bound = HALF_STEP[q.dtype] * want.abs() + (2 * weight + chain) * size + 1e-37
    lists = [pages]
    if long and q.dtype == BF16:
        lists.append(torch.cat((pages, torch.full((1 + 90000000 // (rows * nq // nkv * nkv * hd * page),), -1, dtype=torch.int32, device="cuda"))))
    for these in lists:
        args = (q, k, v, table, ints(lens), these, ints([P]), None if starts is None else ints(starts), scale)
        got = lib.hsd_prefix_attention(*args)
        off = (got.double().cpu() - want).abs()
        assert bool((off <= bound)[~none].all()), (float((off / bound)[~none].max()), int((off > bound)[~none].sum()))
        assert bool((got.cpu()[none] == 0).all())
        into = torch.full_like(q, 7.0)
        assert lib.hsd_prefix_attention(*args, out=into) is into
        assert torch.equal(into[~none.cuda()], got[~none.cuda()]) and bool((into[none.cuda()] == 7.0).all())      # sums in a fixed order
    return got


def prefix_cache(g, batch, nkv, hd, page, P, own, dtype, order="head"):
    """A table whose whole pages below P are no pages at all, and the prefix's pages."""
    per_seq = -(-(P + own) // page)
    k, v, table = cache(g, batch, nkv, hd, page, per_seq, dtype, order, spare=-(-P // page) + 2)
    used = set(table.flatten().tolist())
    free = [p for p in range(k.shape[1]) if p not in used]
    table[:, :P // page] = -7
    pages = ints(free[:max(1, -(-P // page))][::-1])
    return k, v, table, pages


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("nq,nkv", [(1, 1), (8, 2), (7, 1), (40, 2)])
@pytest.mark.parametrize("P", [1, 16, 45, 200])
def test_prefix_attention_of_one_row_each(lib, dtype, hd, nq, nkv, P):
    g = gen(hd + nq + P)
    k, v, table, pages = prefix_cache(g, 7, nkv, hd, 16, P, 60, dtype)
    lens = [P + 1, P, P + 17, 0, P + 60, -1, max(1, P - 3)]
    check_prefix(lib, randn(g, 7, nq, hd, dtype=dtype, std=1.5), k, v, table, lens, pages, P)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("P", [33, 300])
def test_prefix_attention_of_several_rows(lib, dtype, hd, P):
    """One to many rows a sequence, sequences without rows, shorter than their rows, rows in front of the first and behind the last."""
    g = gen(hd + P)
    n = [1, 9, 0, 4, 40, 3, 2]
    starts = [2]
    for x in n:
        starts.append(starts[-1] + x)
    k, v, table, pages = prefix_cache(g, 7, 2, hd, 16, P, 70, dtype)
    lens = [P + 5, P + 9, P + 3, P + 2, P + 70, 2, P - 1]
    check_prefix(lib, randn(g, starts[-1] + 3, 6, hd, dtype=dtype), k, v, table, lens, pages, P, starts)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("page,order", [(1, "head"), (3, "token"), (8, "token"), (24, "head"), (64, "token"), (128, "head")])
def test_prefix_attention_over_pages_of_any_size(lib, dtype, page, order):
    g = gen(page)
    for P in (5, 131):
        k, v, table, pages = prefix_cache(g, 30, 2, 64, page, P, 40, dtype, order)
        lens = [P + 1 + (i * 7) % 40 for i in range(30)]
        check_prefix(lib, randn(g, 30, 8, 64, dtype=dtype), k, v, table, lens, pages, P)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("batch,nq,nkv,P,own", [(1, 4, 1, 9001, 40), (2, 8, 8, 5000, 300), (40, 8, 2, 3001, 20), (70, 4, 1, 2500, 90), (300, 2, 1, 1500, 5)])
def test_prefix_attention_is_joined_where_it_is_divided(lib, dtype, batch, nq, nkv, P, own):
    g = gen(P)
    k, v, table, pages = prefix_cache(g, batch, nkv, 128, 16, P, own, dtype)
    lens = [P + 1 + (i * 13) % own for i in range(batch)]
    check_prefix(lib, randn(g, batch, nq, 128, dtype=dtype, std=2.0), k, v, table, lens, pages, P)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_prefix_attention_without_a_prefix_and_with_more_than_its_pages(lib, dtype):
    g = gen(3)
    k, v, table, pages = prefix_cache(g, 20, 1, 64, 16, 32, 50, dtype)
    q = randn(g, 20, 4, 64, dtype=dtype)
    table[:, :2] = table[:, 2:4]
    for P in (0, -5):
        got = check_prefix(lib, q, k, v, table, [i * 4 for i in range(20)], pages, P)
        assert bool((got[0] == 0).all())
    check_prefix(lib, q, k, v, table, [40 + i for i in range(20)], pages, 1000, long=False)           # 32 positions of the prefix
    long = ints(torch.arange(10).repeat(2).tolist())                                     # a prefix past the sequences' room
    check_prefix(lib, q, k, v, table, [200 + 9 * i for i in range(20)], long, 290)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_prefix_attention_reads_nothing_that_is_not_there(lib, dtype):
    g = gen(5)
    P, batch = 75, 36
    k, v, table, pages = prefix_cache(g, batch, 2, 64, 16, P, 40, dtype)
    lens = [P + 1 + i for i in range(34)] + [0, 70]
    q = randn(g, batch, 8, 64, dtype=dtype)
    args = (table, ints(lens), pages, ints([P]))
    want = lib.hsd_prefix_attention(q, k, v, *args)
    for bad in (float("nan"), float("inf"), torch.finfo(dtype).min):
        k2, v2 = torch.full_like(k, bad), torch.full_like(v, bad)
        for i, n in enumerate(lens):
            for p in range(n):
                at = int(pages[p // 16]) if p < P else int(table[i, p // 16])
                k2[:, at, p % 16], v2[:, at, p % 16] = k[:, at, p % 16], v[:, at, p % 16]
        for p in range(P):
            k2[:, pages[p // 16], p % 16], v2[:, pages[p // 16], p % 16] = k[:, pages[p // 16], p % 16], v[:, pages[p // 16], p % 16]
        assert torch.equal(want, lib.hsd_prefix_attention(q, k2, v2, *args))
    pages[1], pages[3], table[0, 5], table[3, 4] = -1, k.shape[1], 1 << 30, -5            # pages that are none: absent
    check_prefix(lib, q, k, v, table, lens, pages, P)
    pages[:] = -1
    check_prefix(lib, q, k, v, table, lens, pages, P)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_prefix_attention_scales(lib, dtype, scale):
    g = gen(7)
    k, v, table, pages = prefix_cache(g, 40, 1, 64, 16, 400, 30, dtype)
    check_prefix(lib, randn(g, 40, 4, 64, dtype=dtype), k, v, table, [401 + i % 30 for i in range(40)], pages, 400, scale=scale)


@pytest.mark.parametrize("rows", [3, 50])
def test_prefix_attention_keeps_nan_to_its_rows(lib, rows):
    g = gen(8)
    for dtype in (BF16, FP32):
        k, v, table, pages = prefix_cache(g, rows, 1, 64, 16, 600, 20, dtype)
        q = randn(g, rows, 2, 64, dtype=dtype)
        q[0, 1, 3] = float("nan")
        v[0, table[1, 600 // 16], 600 % 16, 0] = float("inf")
        got = lib.hsd_prefix_attention(q, k, v, table, ints([605] * rows), pages, ints([600]))
        assert bool(got[0, 1].isnan().all()) and bool(got[0, 0].isfinite().all()) and bool(got[2:].isfinite().all())
        assert not bool(got[1, :, 0].isfinite().any()) and bool(got[1, :, 1:].isfinite().all())


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("hd,page", [(32, 16), (64, 3), (128, 16)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_prefix_attention_keeps_new_keys_and_values_to_the_rows_that_see_them(lib, dtype, hd, page, bad):
    """A new token's key or value that is not finite: rows in front of it do not see it."""
    g, P, batch = gen(hd), 37, 12
    n = [1 + i % 9 for i in range(batch)]
    starts = [sum(n[:i]) for i in range(batch + 1)]
    lens = [P + n[i] + 5 * i for i in range(batch)]
    k, v, table, pages = prefix_cache(g, batch, 2, hd, page, P, 80, dtype)
    q = randn(g, starts[-1], 8, hd, dtype=dtype)
    args = (table, ints(lens), pages, ints([P]), ints(starts))
    want = lib.hsd_prefix_attention(q, k, v, *args)
    for pool in (k, v):
        keep, blind = pool.clone(), []
        for b in range(batch):
            first = n[b] // 2                                               # rows from here on see a bad token, the last one two
            for r in {first, n[b] - 1}:
                at = lens[b] - n[b] + r
                pool[:, table[b, at // page], at % page, hd // 3] = bad
            blind += [starts[b] + r for r in range(first)]
        got = lib.hsd_prefix_attention(q, k, v, *args)
        assert torch.equal(got[blind], want[blind])
        sees = [r for r in range(starts[-1]) if r not in blind]
        if pool is v:
            assert not bool(got[sees][:, :, hd // 3].isfinite().any())
        elif bad != bad:
            assert bool(got[sees].isnan().all())
        pool.copy_(keep)


@pytest.mark.parametrize("rows", [3, 60])
def test_prefix_attention_follows_its_lists_when_replayed_and_on_other_streams(lib, rows):
    g = gen(11)
    k, v, table, pages = prefix_cache(g, rows, 2, 64, 16, 1000, 100, BF16)
    q, lens, P = randn(g, rows, 8, 64, dtype=BF16), ints([0] * rows), ints([0])
    starts = ints(list(range(rows + 1)))
    other_q = randn(g, rows, 8, 64, dtype=BF16)
    lib.hsd_prefix_attention(q, k, v, table, lens, pages, P, starts)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x in (q, other_q):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(lib.hsd_prefix_attention(x, k, v, table, lens, pages, P, starts))
        graphs.append(graph)
    for prefix, shift in ((1000, 0), (992, 1), (3, 0), (0, 0)):
        values = [prefix + 1 + (i * 17) % 90 for i in range(rows)]
        lens.copy_(ints(values))
        P.copy_(ints([prefix]))
        starts.copy_(ints([max(0, i - shift) for i in range(rows + 1)]))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for x, out in zip((q, other_q), outs):
            assert torch.equal(out, lib.hsd_prefix_attention(x, k, v, table, ints(values), pages, ints([prefix]), starts.clone()))
    lens, P = ints([1001 + i for i in range(rows)]), ints([1000])
    want = [lib.hsd_prefix_attention(x, k, v, table, lens, pages, P) for x in (q, other_q)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(20):
        for i, (x, s) in enumerate(zip((q, other_q), streams)):
            with torch.cuda.stream(s):
                got[i].append(lib.hsd_prefix_attention(x, k, v, table, lens, pages, P))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(y, want[i]) for y in got[i])


def test_prefix_attention_of_one_table_is_the_attention_by_sequence(lib):
    """Tables that name the prefix's pages themselves: what hsd_paged_attention gives, to the rounding of the sums."""
    g = gen(12)
    for dtype in (BF16, FP32):
        P, batch = 512, 33
        k, v, table, pages = prefix_cache(g, batch, 2, 128, 16, P, 64, dtype)
        table[:, :P // 16] = pages
        lens, q = ints([P + 1 + i for i in range(batch)]), randn(g, batch, 8, 128, dtype=dtype)
        a, b = lib.hsd_prefix_attention(q, k, v, table, lens, pages, ints([P])), lib.hsd_paged_attention(q, k, v, table, lens)
        size = v.abs().max()
        assert bool(((a.double() - b.double()).abs() <= 2 * HALF_STEP[dtype] * b.double().abs() + 2.0 ** -15 * size).all())


def test_prefix_attention_far_into_a_large_pool(lib):
    """Places past 2^31 elements and 2^32 bytes of a pool."""
    g = gen(13)
    n_pages = (1 << 31) // (16 * 128) + 40
    k, v = (torch.empty(1, n_pages, 16, 128, dtype=BF16, device="cuda") for _ in range(2))
    pages = ints([n_pages - 1, 3, n_pages - 30])
    table = ints([[-1, -1, n_pages - 2, n_pages - 3], [-1, -1, 7, n_pages - 5]] * 12)
    for p in pages.tolist() + table[table >= 0].flatten().tolist():
        k[0, p], v[0, p] = randn(g, 16, 128, dtype=BF16), randn(g, 16, 128, dtype=BF16)
    check_prefix(lib, randn(g, 24, 4, 128, dtype=BF16), k, v, table, [45 + i % 19 for i in range(24)], pages, 44)


@pytest.mark.parametrize("nq,nkv", [(32, 1), (14, 2), (80, 2), (64, 1), (65, 1)])
@pytest.mark.parametrize("rows", [4, 19, 70])
def test_prefix_attention_of_query_tiles_that_are_not_full(lib, rows, nq, nkv):
    """Groups that divide a tile of 128 queries or do not, one query tile, two, an odd number of them; groups past a half of one."""
    g = gen(rows + nq)
    k, v, table, pages = prefix_cache(g, rows, nkv, 128, 16, 150, 20, BF16)
    check_prefix(lib, randn(g, rows, nq, 128, dtype=BF16), k, v, table, [151 + i % 20 for i in range(rows)], pages, 150)


def prefix_in_64_bits(q, k, v, pages, P, scale):
    out, group, hd = torch.empty(q.shape, dtype=torch.float64, device="cuda"), q.shape[1] // k.shape[0], q.shape[2]
    for h in range(k.shape[0]):
        kh, vh = (x[h][pages.long()].reshape(-1, hd)[:P].double() for x in (k, v))
        for r in range(0, q.shape[0], 100):
            out[r:r + 100, h * group:(h + 1) * group] = torch.softmax(q[r:r + 100, h * group:(h + 1) * group].double() @ kh.T * scale, dim=-1) @ vh
    return out


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("grows", [False, True])
def test_prefix_attention_adds_long_chains_in_fp32(lib, hd, grows):
    """Several chains a CTA.  Means of 1 and its neighbour lie about their middle, where a small loss rounds down what should be rounded up; and
    scores that grow along the keys, so that a row's reference moves between the chains."""
    g, rows, P = gen(hd), 500, 40000
    k = randn(g, 1, P // 16, 16, hd, dtype=BF16)
    v = (1 + 2.0 ** -7 * torch.randint(0, 2, k.shape, generator=g, device="cuda")).to(BF16)
    q = randn(g, rows, 8, hd, dtype=BF16, std=0.3)
    if grows:
        k[0, :, :, 0] = torch.linspace(0, 20, P // 16, device="cuda")[:, None].to(BF16)
        q[:, :, 0] = 30.0
    pages = torch.randperm(P // 16, generator=g, device="cuda").to(torch.int32).contiguous()
    if grows:
        pages = torch.arange(P // 16, dtype=torch.int32, device="cuda")
    scale = hd ** -0.5
    got = lib.hsd_prefix_attention(q, k, v, ints([[0]]).expand(rows, 1).contiguous(), ints([P] * rows), pages, ints([P])).double()
    want = prefix_in_64_bits(q, k, v, pages, P, scale)
    # a chain: 256 products, of which each may cut off 2^-23; chains and parts: some twenty additions and the quotient; the weights' sum: a CTA's 4300
    # keys in four turns, nearest (eight deviations of 2^-24 / sqrt(3)); a weight counts by the values' difference, 2^-7, alone
    most = float((q.double().abs().amax(dim=(0, 1)) * k.double().abs().amax(dim=(0, 1, 2))).sum()) * scale
    bound = 256 * 2.0 ** -23 + 24 * 2.0 ** -24 + 8 / 3 ** 0.5 * 1075 ** 0.5 * 2.0 ** -24 + 2.0 ** -7 * (2.0 ** -15 + (hd + 4) * 2.0 ** -22 * most)
    assert bool(((got - want).abs() <= 2.0 ** -8 + bound * want).all()), float(((got - want).abs() - 2.0 ** -8).max())
    again = lib.hsd_prefix_attention(q, k, v, ints([[0]]).expand(rows, 1).contiguous(), ints([P] * rows), pages, ints([P])).double()
    assert torch.equal(got, again)


# ------------------------------------------------------------------------------------------------ together
class Layer:
    """One attention layer of a decoder with 8-bit weights and norms of queries and keys, over continuations of one prompt."""
    d, nq, nkv, hd, page = 512, 8, 2, 64, 16

    def __init__(self, lib, seed, batch, P, own):
        g = gen(seed)
        self.lib, self.P = lib, P
        heads = self.nq + 2 * self.nkv
        self.qkv = lib.hsd_quantize_rows(randn(g, heads * self.hd, self.d, dtype=BF16, std=self.d ** -0.5))
        self.out = lib.hsd_quantize_rows(randn(g, self.d, self.nq * self.hd, dtype=BF16, std=self.d ** -0.5))
        self.gains = [1 + randn(g, self.hd, std=0.2).to(BF16) for _ in range(2)]
        self.rope = lib.rope_table(P + own, self.hd)
        self.k, self.v, self.table, self.pages = prefix_cache(g, batch, self.nkv, self.hd, self.page, P, own, BF16)
        self.prefix = ints([P])
        # room behind the prefix in the list, so that its sums go by tensor memory
        self.pages = torch.cat((self.pages, torch.full((3000,), -1, dtype=torch.int32, device="cuda")))

    def step(self, x, before, after, starts):
        """x [rows, d] -> (rows of q, k and v, queries, attention, output)."""
        lib = self.lib
        qkv = lib.hsd_gemm_w8(x, *self.qkv)
        q = lib.hsd_kv_append_norm(qkv.view(len(x), -1, self.hd), *self.gains, 1e-6, self.k, self.v, self.table, before, self.rope, starts)
        att = lib.hsd_prefix_attention(q, self.k, self.v, self.table, after, self.pages, self.prefix, starts)
        return qkv, q, att, lib.hsd_gemm_w8(att.view(len(x), -1), *self.out, BF16)


def test_a_layer_of_continuations_of_one_prompt(lib):
    """The calls of a step as they follow one another, each against 64 bits on what the one before gave; steps of one to three rows."""
    batch, P = 24, 100
    layer, lens = Layer(lib, 5, batch, P, 40), [P + i % 7 for i in range(batch)]
    for turn in range(3):
        n = [1 + (i + turn) % 3 for i in range(batch)]
        starts = [sum(n[:i]) for i in range(batch + 1)]
        x = randn(gen(turn), starts[-1], layer.d, dtype=BF16)
        after = [a + b for a, b in zip(lens, n)]
        keep = layer.k.clone(), layer.v.clone()
        qkv, q, att, y = layer.step(x, ints(lens), ints(after), ints(starts))
        assert torch.equal(qkv, check_w8(lib, x, *layer.qkv))
        k1, v1 = layer.k.clone(), layer.v.clone()
        layer.k.copy_(keep[0]), layer.v.copy_(keep[1])
        found = append64(qkv.view(len(x), -1, layer.hd), layer.gains, 1e-6, layer.table, lens, layer.rope, starts, layer.nkv, (layer.k.shape[1], layer.page))
        assert len(found) == len(x)
        for r, (pg, t, qy, ky, vx, size) in found.items():
            assert bool(((q[r].double().cpu() - qy).abs() <= 2.0 ** -8 * qy.abs() + 18 * 2.0 ** -24 * size[:layer.nq] + 1e-37).all())
            layer.k[:, pg, t], layer.v[:, pg, t] = k1[:, pg, t], v1[:, pg, t]
        assert torch.equal(layer.k, k1) and torch.equal(layer.v, v1)                      # nothing else was written
        assert torch.equal(att, check_prefix(lib, q, layer.k, layer.v, layer.table, after, layer.pages, P, starts, long=False))
        assert torch.equal(y, check_w8(lib, att.view(len(x), -1), *layer.out, BF16))
        lens = after


def test_a_captured_layer_follows_its_inputs_and_two_at_once(lib):
    batch, P = 24, 100
    layers = [Layer(lib, 6 + i, batch, P, 40) for i in range(2)]
    xs = [randn(gen(i), batch, Layer.d, dtype=BF16) for i in range(2)]
    before, after = ints([P] * batch), ints([P + 1] * batch)
    for layer, x in zip(layers, xs):
        layer.step(x, before, after, None)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for layer, x in zip(layers, xs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(layer.step(x, before, after, None)[3])
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(6):
        before.copy_(ints([P + turn] * batch)), after.copy_(ints([P + turn + 1] * batch))
        for i, x in enumerate(xs):
            x.copy_(randn(gen(10 + 2 * turn + i), batch, Layer.d, dtype=BF16))
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for layer, x, out in zip(layers, xs, outs):
            assert torch.equal(out, layer.step(x, before, after, None)[3])


# ------------------------------------------------------------------------------------------------ on tensor memory
def with_room(pages, keys=400000):
    """A list with room for many keys behind the prefix's end, so that the call's sums over the prefix go by tensor memory."""
    return torch.cat((pages, torch.full((keys // 16,), -1, dtype=torch.int32, device="cuda")))


@pytest.mark.parametrize("hd", [64, 128])
def test_prefix_attention_on_tensor_memory_reads_nothing_that_is_not_there(lib, hd):
    g, P, batch = gen(hd), 75, 36
    k, v, table, pages = prefix_cache(g, batch, 2, hd, 16, P, 40, BF16)
    lens = [P + 1 + i for i in range(34)] + [0, 70]
    q = randn(g, batch, 8, hd, dtype=BF16)
    args = (table, ints(lens), with_room(pages), ints([P]))
    want = lib.hsd_prefix_attention(q, k, v, *args)
    for bad in (float("nan"), float("inf"), torch.finfo(BF16).min):
        k2, v2 = torch.full_like(k, bad), torch.full_like(v, bad)
        for i, n in enumerate(lens):
            for p in range(P, n):
                at = int(table[i, p // 16])
                k2[:, at, p % 16], v2[:, at, p % 16] = k[:, at, p % 16], v[:, at, p % 16]
        for p in range(P):
            k2[:, pages[p // 16], p % 16], v2[:, pages[p // 16], p % 16] = k[:, pages[p // 16], p % 16], v[:, pages[p // 16], p % 16]
        assert torch.equal(want, lib.hsd_prefix_attention(q, k2, v2, *args))


@pytest.mark.parametrize("rows", [50, 130])
def test_prefix_attention_on_tensor_memory_keeps_nan_to_its_rows(lib, rows):
    g = gen(rows)
    k, v, table, pages = prefix_cache(g, rows, 1, 64, 16, 600, 20, BF16)
    q = randn(g, rows, 2, 64, dtype=BF16)
    q[0, 1, 3], q[rows - 1, 0, 9] = float("nan"), float("inf")
    args = (table, ints([605] * rows), with_room(pages), ints([600]))
    got = lib.hsd_prefix_attention(q, k, v, *args)
    assert bool(got[0, 1].isnan().all()) and bool(got[0, 0].isfinite().all()) and bool(got[1:-1].isfinite().all()) and bool(got[-1, 0].isnan().all())
    v[0, pages[7], 3, 11] = float("nan")                                    # seen by all rows
    assert bool(lib.hsd_prefix_attention(q, k, v, *args)[:, :, 11].isnan().all())
    v[0, pages[7], 3, 11], k[0, pages[9], 2, 5] = 0, float("nan")
    assert bool(lib.hsd_prefix_attention(q, k, v, *args).isnan().all())


def test_prefix_attention_on_tensor_memory_follows_its_lists_when_replayed_and_on_two_streams(lib):
    g, rows = gen(14), 70
    k, v, table, pages = prefix_cache(g, rows, 2, 128, 16, 5000, 100, BF16)
    qs, lens, P = [randn(g, rows, 8, 128, dtype=BF16) for _ in range(2)], ints([0] * rows), ints([0])
    room = with_room(pages)
    lib.hsd_prefix_attention(qs[0], k, v, table, lens, room, P)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x in qs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(lib.hsd_prefix_attention(x, k, v, table, lens, room, P))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in qs]
    for prefix in (5000, 4992, 64, 1, 0, 2049):
        values = [prefix + 1 + (i * 17) % 90 for i in range(rows)] if prefix >= 4992 else [prefix] * rows
        lens.copy_(ints(values)), P.copy_(ints([prefix]))
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for x, out in zip(qs, outs):
            assert torch.equal(out, lib.hsd_prefix_attention(x, k, v, table, ints(values), room, ints([prefix])))


@pytest.mark.parametrize("order,page", [("head", 8), ("token", 24), ("token", 64), ("head", 256)])
@pytest.mark.parametrize("hd", [64, 128])
def test_prefix_attention_on_tensor_memory_over_pages_of_any_eights(lib, order, page, hd):
    g = gen(page)
    for P in (63, 64, 65, 700):
        k, v, table, pages = prefix_cache(g, 9, 2, hd, page, P, 30, BF16, order)
        check_prefix(lib, randn(g, 9, 12, hd, dtype=BF16), k, v, table, [P + 1 + i for i in range(9)], pages, P)


def test_prefix_attention_takes_a_batch_of_thousands(lib):
    g, batch, P = gen(15), 4096, 7
    for dtype in (BF16, FP32):
        k, v, table = cache(g, batch, 1, 32, 4, 4, dtype)
        pages = ints([batch * 4, batch * 4 + 1])
        spare = [p for p in range(k.shape[1]) if p not in set(table.flatten().tolist())]
        pages = ints(spare[:2])
        lens, q = ints([P + 1 + i % 9 for i in range(batch)]), randn(g, batch, 1, 32, dtype=dtype)
        for t in (k, v):                                                    # the prefix's last page is half each sequence's own
            t[:, table[:, 1].long(), :3] = t[:, pages[1].long(), :3][:, None]
        table[:, 0] = pages[0]
        a, b = lib.hsd_prefix_attention(q, k, v, table, lens, pages, ints([P])), lib.hsd_paged_attention(q, k, v, table, lens)
        assert bool(((a.double() - b.double()).abs() <= 2 * HALF_STEP[dtype] * b.double().abs() + 2.0 ** -18 * v.abs().max()).all())


# ------------------------------------------------------------------------------------------------ how exact the sums on tensor memory are
def launches(lib, call):
    before = lib.hsd_kernel_launches()
    out = call()
    return out, lib.hsd_kernel_launches() - before


@pytest.mark.parametrize("hd", [64, 128])
def test_prefix_attention_on_tensor_memory_keeps_all_bits_of_its_weights(lib, hd):
    """Differences of the weights of two keys whose scores are nearly the same: what a weight of fewer bits is off by stands out in them."""
    g, rows, pairs = gen(hd), 64, 32
    q, k = torch.zeros(rows, 8, hd, device="cuda"), torch.zeros(1, 4, 16, hd, device="cuda")
    # scores in whole 2^-13s below 2^4: exact in any order of their sum
    q[..., 0], q[..., 1] = (1 + torch.randint(0, 16, (rows, 8), generator=g, device="cuda") / 16), 2.0 ** -8
    key = k.view(2 * pairs, hd)
    key[:, 0] = (torch.randint(0, 16, (pairs,), generator=g, device="cuda") / 16).repeat_interleave(2)
    key[1::2, 1] = 2.0 ** -5 * torch.randint(1, 4, (pairs,), generator=g, device="cuda")
    v = torch.zeros(1, 4, 16, hd, device="cuda")
    for i in range(pairs):                                                  # column i: the pair's first weight less its second
        v.view(2 * pairs, hd)[2 * i, i], v.view(2 * pairs, hd)[2 * i + 1, i] = 1, -1
    q, k, v = q.to(BF16), k.to(BF16), v.to(BF16)
    args = (ints([[0]]).expand(rows, 1).contiguous(), ints([64] * rows), with_room(ints([0, 1, 2, 3]), 1 << 23), ints([64]), None, 1.0)
    got, n = launches(lib, lambda: lib.hsd_prefix_attention(q, k, v, *args))
    assert n == 3                                                           # on tensor memory
    w = torch.softmax(q.double() @ key.to(BF16).double().T, dim=-1)
    want = w @ v.double().view(2 * pairs, hd)
    # an exponential is off by 2^-22 of itself, its argument (below 4) by half a place, 2^-22, twice each; the four products of 16 keys' high parts may cut off 2^-23 of
    # the largest weight each; the rest (sum of the weights, quotient: factors of the difference) is less than one of these
    bound = HALF_STEP[BF16] * want.abs() + w.amax(dim=-1, keepdim=True) * (2 * 2.0 ** -22 * (1 + math.log(2)) + 5 * 2.0 ** -23)
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())


# ------------------------------------------------------------------------------------------------ lists that name more rows than there are
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("cut", [1, 6, 11])
def test_prefix_attention_of_a_list_that_names_more_rows(lib, dtype, cut):
    """The rows that are there see what they would see in the whole call, as an append of the same list places them."""
    g, P = gen(cut), 50
    n = [2, 5, 9, 4]
    starts = [sum(n[:i]) for i in range(5)]
    k, v, table, pages = prefix_cache(g, 4, 2, 64, 16, P, 40, dtype)
    lens = [P + 2, P + 20, P + 9, P + 30]
    q = randn(g, starts[-1], 8, 64, dtype=dtype)
    whole = check_prefix(lib, q, k, v, table, lens, pages, P, starts)
    part = check_prefix(lib, q[:-cut].contiguous(), k, v, table, lens, pages, P, starts)
    size = v.abs().max().double()
    assert bool(((part.double() - whole[:-cut].double()).abs() <= 2 * HALF_STEP[dtype] * whole[:-cut].double().abs() + 2.0 ** -15 * size).all())
    # rows in front of the call's first: the first three of a sequence
    shifted = [s - 3 for s in starts]
    late = lib.hsd_prefix_attention(q[3:].contiguous(), k, v, table, ints(lens), pages, ints([P]), ints(shifted))
    assert bool(((late.double() - whole[3:].double()).abs() <= 2 * HALF_STEP[dtype] * whole[3:].double().abs() + 2.0 ** -15 * size).all())


# ------------------------------------------------------------------------------------------------ sizes next to 2^31
@pytest.mark.parametrize("R,N", [(1, (1 << 31) - 300), ((1 << 31) - 300, 1)])
def test_products_of_sizes_next_to_their_limit(lib, R, N):
    K, g = 16, gen(1)
    a, w = (torch.ones(n, K, dtype=torch.int8, device="cuda") for n in (R, N))
    rows, cols = torch.ones(R, device="cuda"), torch.ones(N, device="cuda")
    for x in (a, w):
        x[-1000:] = torch.randint(-128, 128, x[-1000:].shape, generator=g, device="cuda").to(torch.int8)
    out = lib.hsd_gemm_w8(a, w, cols, BF16, a_scales=rows)
    few = w if R == 1 else a                                                # the long one; the other has one row
    one = (a if R == 1 else w).float()[0]
    long, count = out.view(-1), few.shape[0]
    assert torch.equal(long[-1000:], (few[-1000:].float() @ one).to(BF16))
    first = one.sum().to(BF16)
    for i in range(0, count - 1000, 1 << 28):
        assert bool((long[i:min(i + (1 << 28), count - 1000)] == first).all())


# ------------------------------------------------------------------------------------------------ appends where the rows of a CTA change
@pytest.mark.parametrize("rows,nq,nkv", [(592, 3, 1), (593, 3, 1), (1184, 2, 1), (1185, 2, 1), (2368, 1, 1), (2369, 1, 1), (149, 130, 8), (296, 130, 8), (297, 130, 8), (593, 60, 20)])
def test_appends_where_the_rows_of_a_cta_change(lib, rows, nq, nkv):
    g, batch = gen(rows), 5
    starts = [rows * i // batch for i in range(batch + 1)]
    before = [3 * i for i in range(batch)]
    longest = max(b + starts[i + 1] - starts[i] for i, b in enumerate(before))
    k, v, table = cache(g, batch, nkv, 32, 16, -(-longest // 16), BF16)
    qkv, rope = randn(g, rows, nq + 2 * nkv, 32, dtype=BF16), lib.rope_table(longest, 32)
    assert len(check_append(lib, qkv, [randn(g, 32), randn(g, 32)], 1e-6, k, v, table, before, rope, starts)) == rows
    # without norms: the same as in pieces of a sequence's rows, which a call of few rows takes otherwise
    whole = lib.hsd_kv_append(qkv, k, v, table, ints(before), rope, ints(starts))
    kept = k.clone(), v.clone()
    k.zero_(), v.zero_()
    for b in range(batch):
        for r in range(starts[b], starts[b + 1], 100):
            n = min(100, starts[b + 1] - r)
            part = lib.hsd_kv_append(qkv[r:r + n], k, v, table[b:b + 1], ints([before[b] + r - starts[b]]), rope, ints([0, n]))
            assert torch.equal(part, whole[r:r + n])
    used = torch.zeros(k.shape[1], 16, dtype=torch.bool)
    for b in range(batch):
        for p in range(before[b], before[b] + starts[b + 1] - starts[b]):
            used[int(table[b, p // 16]), p % 16] = True
    used = used.cuda()
    assert torch.equal(k[:, used], kept[0][:, used]) and torch.equal(v[:, used], kept[1][:, used])


# ------------------------------------------------------------------------------------------------ CTAs that go from one query tile to two
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows,nq,nkv,P", [(65, 8, 2, 10000), (65, 640, 160, 700), (65, 600, 150, 130), (33, 512, 64, 1000)])
def test_prefix_attention_of_sets_with_one_query_tile_and_with_two(lib, hd, rows, nq, nkv, P):
    """Rows that make a set of two query tiles and one of one, for each key head: CTAs go from the end of the one to the other."""
    g = gen(rows + nq + hd)
    k, v = (randn(g, nkv, -(-P // 16), 16, hd, dtype=BF16) for _ in range(2))
    q, pages = randn(g, rows, nq, hd, dtype=BF16), torch.randperm(-(-P // 16), generator=g, device="cuda").to(torch.int32)
    args = (ints([[0]] * rows), ints([P] * rows), with_room(pages, 1 << 22), ints([P]))
    got, n = launches(lib, lambda: lib.hsd_prefix_attention(q, k, v, *args))
    assert n == 3
    scale = hd ** -0.5
    want, size = prefix_in_64_bits(q, k, v, pages, P, scale), prefix_in_64_bits(q, k, v.abs(), pages, P, scale)
    most = float((q.double().abs().amax(dim=(0, 1)) * k.double().abs().amax(dim=(0, 1, 2))).sum()) * scale
    weight = (hd + 4) * 2.0 ** -23 * most + 2.0 ** -21 + (P / 8 + 64) * 2.0 ** -24
    assert bool(((got.double() - want).abs() <= HALF_STEP[BF16] * want.abs() + (2 * weight + 12 * 2.0 ** -23) * size).all())
    for _ in range(10):
        assert torch.equal(got, lib.hsd_prefix_attention(q, k, v, *args))


# ------------------------------------------------------------------------------------------------ which kernels a call takes
def kernels_of(lib, dtype=BF16, hd=64, page=16, order="head", rows=40, nq=8, nkv=2, scale=None, room=True):
    g = gen(1)
    k, v, table, pages = prefix_cache(g, rows, nkv, hd, page, 100, 20, dtype, order)
    args = (randn(g, rows, nq, hd, dtype=dtype), k, v, table, ints([101] * rows), with_room(pages, 1 << 24) if room else pages, ints([100]), None, scale)
    return launches(lib, lambda: lib.hsd_prefix_attention(*args))[1]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("call", [{}, dict(order="token"), dict(page=8), dict(page=24, order="token"), dict(page=24), dict(page=64, order="token"), dict(page=128), dict(page=256), dict(rows=4),
                                  dict(nq=32, nkv=1), dict(nq=14, nkv=2), dict(nq=80, nkv=2), dict(nq=64, nkv=1), dict(nq=7, nkv=1, rows=70), dict(rows=300, nq=2, nkv=1), dict(scale=4.0)])
def test_prefix_attention_takes_tensor_memory(lib, hd, call):
    """The kernel for the prefix, the one for own keys, the join: what tests with room in the list of pages take for granted."""
    assert kernels_of(lib, hd=hd, **call) == 3


@pytest.mark.parametrize("call", [dict(room=False), dict(dtype=FP32), dict(hd=32), dict(page=3), dict(page=12), dict(scale=0.0), dict(scale=-0.3), dict(nq=65, nkv=1), dict(rows=3, nq=8, nkv=2)])
def test_prefix_attention_takes_sets_of_queries(lib, call):
    assert kernels_of(lib, **call) == 2


def test_layers_and_long_chains_take_tensor_memory(lib):
    layer = Layer(lib, 5, 24, 100, 40)
    q = randn(gen(1), 24, layer.nq, layer.hd, dtype=BF16)
    assert launches(lib, lambda: lib.hsd_prefix_attention(q, layer.k, layer.v, layer.table, ints([101] * 24), layer.pages, layer.prefix))[1] == 3
    k, pages = randn(gen(2), 1, 2500, 16, 64, dtype=BF16), ints(list(range(2500)))
    assert launches(lib, lambda: lib.hsd_prefix_attention(randn(gen(3), 500, 8, 64, dtype=BF16), k, k, ints([[0]] * 500), ints([40000] * 500), pages, ints([40000])))[1] == 3
