"""The operators of a caller's own drafter against plain implementations in 64 bits: lengths from none to many pages, odd sizes,
strides, pages in any order, masks that leave nothing, values that are not finite where nothing may read them.

Tolerances count roundings: half a step of the output's type, 2^-24 for each fp32 operation in a sum, 2^-23 where the tensor cores'
adders may cut off instead of rounding."""
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


# ------------------------------------------------------------------------------------------------ attention
def attention64(q, k_pool, v_pool, table, lens, scale):
    """(out, sum of weights times |v|, the largest sum of |q||k|), all in 64 bits."""
    b, nq, hd = q.shape
    nkv, n_pages, page, _ = k_pool.shape
    out, size, most = (torch.zeros(b, nq, n, dtype=torch.float64) for n in (hd, hd, 1))
    for i, n in enumerate(lens):
        n = min(max(n, 0), table.shape[1] * page)
        where = [(int(table[i, p // page]), p % page) for p in range(n)]
        where = [(a, t) for a, t in where if 0 <= a < n_pages]
        if not where:
            continue
        a, t = (torch.tensor(x, device=q.device) for x in zip(*where))
        for h in range(nq):
            k, v = (x[h * nkv // nq][a, t].double().cpu() for x in (k_pool, v_pool))
            x = q[i, h].double().cpu()
            w = torch.softmax(k @ x * scale, dim=0)
            out[i, h], size[i, h], most[i, h] = w @ v, w @ v.abs(), (k.abs() @ x.abs()).max() * abs(scale)
    return out, size, most


def check_attention(lib, q, k_pool, v_pool, table, lens, scale=None, **more):
    got = lib.hsd_paged_attention(q, k_pool, v_pool, table, ints(lens), scale, **more)
    hd = q.shape[2]
    want, size, most = attention64(q, k_pool, v_pool, table.cpu(), lens, hd ** -0.5 if scale is None else scale)
    # a score's sum has hd products and a scaling, its exponential a few roundings more (relative 2^-22); a weight is off by as much
    # both above and below the line; tiles are added one after the other; bf16 weights keep 16 bits
    weight = (hd + 4) * 2.0 ** -23 * most + 2.0 ** -21 + (max(lens) / 8 + 64) * 2.0 ** -24 + (2.0 ** -16 if q.dtype == BF16 else 0)
    bound = HALF_STEP[q.dtype] * want.abs() + 2 * weight * size + 1e-37
    off = (got.double().cpu() - want).abs()
    assert bool((off <= bound).all()), (float((off / bound).max()), int((off > bound).sum()))
    return got


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("nq,nkv", [(1, 1), (4, 4), (8, 2), (7, 1), (16, 2), (40, 2)])
def test_attention_of_ragged_lengths(lib, dtype, hd, nq, nkv):
    g = gen(hd + nq)
    lens = [0, 1, 2, 15, 16, 17, 63, 130, 200, -1]
    k, v, table = cache(g, len(lens), nkv, hd, 16, 13, dtype)
    check_attention(lib, randn(g, len(lens), nq, hd, dtype=dtype, std=1.5), k, v, table, lens)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("page,order", [(1, "head"), (3, "token"), (8, "token"), (16, "token"), (24, "head"), (64, "token")])
def test_attention_over_pages_of_any_size(lib, dtype, page, order):
    g = gen(page)
    lens = [97, 5, 96, 33]
    k, v, table = cache(g, 4, 2, 64, page, -(-97 // page), dtype, order)
    check_attention(lib, randn(g, 4, 8, 64, dtype=dtype), k, v, table, lens)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("batch,nq,nkv,longest", [(1, 8, 8, 9000), (1, 4, 1, 20011), (3, 16, 2, 3001), (70, 2, 2, 300)])
def test_attention_is_joined_where_sequences_are_divided(lib, dtype, batch, nq, nkv, longest):
    g = gen(longest)
    lens = [max(1, longest * (i + 1) // batch) for i in range(batch)][::-1]
    k, v, table = cache(g, batch, nkv, 128, 16, -(-longest // 16), dtype)
    q = randn(g, batch, nq, 128, dtype=dtype, std=2.0)
    a = check_attention(lib, q, k, v, table, lens)
    assert torch.equal(a, lib.hsd_paged_attention(q, k, v, table, ints(lens)))             # sums in a fixed order


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attention_reads_nothing_behind_a_length(lib, dtype):
    g = gen(5)
    lens = [19, 0, 40, 1]
    k, v, table = cache(g, 4, 2, 64, 16, 4, dtype)
    q = randn(g, 4, 4, 64, dtype=dtype)
    want = lib.hsd_paged_attention(q, k, v, table, ints(lens))
    for bad in (float("nan"), float("inf"), torch.finfo(dtype).min):
        k2, v2 = torch.full_like(k, bad), torch.full_like(v, bad)
        for i, n in enumerate(lens):
            for p in range(n):
                at = int(table[i, p // 16])
                k2[:, at, p % 16], v2[:, at, p % 16] = k[:, at, p % 16], v[:, at, p % 16]
        assert torch.equal(want, lib.hsd_paged_attention(q, k2, v2, table, ints(lens)))
    assert bool((want[1] == 0).all())


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_attention_pages_out_of_the_pool_are_absent(lib, dtype):
    g = gen(6)
    lens = [64, 64, 1000, 16]                       # the third: more than the table has room for
    k, v, table = cache(g, 4, 2, 32, 16, 4, dtype)
    table[0, 1], table[0, 3], table[1], table[3, 0] = -1, k.shape[1], 1 << 30, -5
    got = check_attention(lib, randn(g, 4, 4, 32, dtype=dtype), k, v, table, lens)
    assert bool((got[1] == 0).all()) and bool((got[3] == 0).all())


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_attention_scales(lib, dtype, scale):
    g = gen(7)
    k, v, table = cache(g, 2, 1, 64, 16, 8, dtype)
    check_attention(lib, randn(g, 2, 4, 64, dtype=dtype), k, v, table, [100, 128], scale)


def test_attention_passes_nan_on(lib):
    g = gen(8)
    for dtype in (BF16, FP32):
        k, v, table = cache(g, 2, 1, 64, 16, 40, dtype)
        q = randn(g, 2, 2, 64, dtype=dtype)
        q[0, 1, 3] = float("nan")
        got = lib.hsd_paged_attention(q, k, v, table, ints([600, 600]))
        assert bool(got[0, 1].isnan().all()) and not bool(got[0, 0].isnan().any()) and not bool(got[1].isnan().any())


def test_attention_takes_a_batch_of_thousands(lib):
    g = gen(9)
    k, v, table = cache(g, 4096, 1, 32, 4, 2, BF16)
    lens = ints([i % 9 for i in range(4096)])
    got = lib.hsd_paged_attention(randn(g, 4096, 1, 32, dtype=BF16), k, v, table, lens)
    assert bool((got[lens == 0] == 0).all()) and bool((got[lens > 0].abs().amax(dim=(1, 2)) > 0).all())
    assert torch.equal(got[lens == 1][:, 0], v[0, table[lens == 1][:, 0].long(), 0])         # one key: its value


def test_attention_far_into_a_large_pool(lib):
    """Places past 2^31 elements and 2^32 bytes of a pool."""
    g = gen(10)
    n_pages = (1 << 31) // (16 * 128) + 40
    k, v = (torch.empty(1, n_pages, 16, 128, dtype=BF16, device="cuda") for _ in range(2))
    table = ints([[n_pages - 1, 3, n_pages - 30], [n_pages - 2, n_pages - 3, 5]])
    for p in table.flatten().tolist():
        k[0, p], v[0, p] = randn(g, 16, 128, dtype=BF16), randn(g, 16, 128, dtype=BF16)
    check_attention(lib, randn(g, 2, 4, 128, dtype=BF16), k, v, table, [48, 41])
    rope = lib.rope_table(64, 128)
    qkv = randn(g, 2, 3, 128)
    lib.hsd_kv_append(qkv, k, v, table, ints([5, 20]), rope)
    assert torch.equal(v[0, n_pages - 1, 5], qkv[0, 2].to(BF16)) and torch.equal(v[0, n_pages - 3, 4], qkv[1, 2].to(BF16))


def test_attention_follows_lengths_when_replayed_and_on_other_streams(lib):
    g = gen(11)
    k, v, table = cache(g, 3, 2, 64, 16, 50, BF16)
    q, lens = randn(g, 3, 4, 64, dtype=BF16), ints([1, 2, 3])
    other_q = randn(g, 3, 4, 64, dtype=BF16)
    lib.hsd_paged_attention(q, k, v, table, lens)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for x in (q, other_q):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(lib.hsd_paged_attention(x, k, v, table, lens))
        graphs.append(graph)
    for values in ([700, 3, 0], [5, 800, 799], [0, 0, 0]):
        lens.copy_(ints(values))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for x, out in zip((q, other_q), outs):
            assert torch.equal(out, lib.hsd_paged_attention(x, k, v, table, ints(values)))
    want = lib.hsd_paged_attention(q, k, v, table, ints([700, 3, 5]))
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = lib.hsd_paged_attention(q, k, v, table, ints([700, 3, 5]))
        torch.cuda.current_stream().synchronize()
    assert torch.equal(got, want)


def shared_pages(g, batch, nkv, n, hd, dtype, values):
    """Pools of one text of n keys, and a table by which every sequence has it."""
    pages = -(-n // 16)
    k = randn(g, nkv, pages, 16, hd, dtype=dtype)
    return k, values(nkv, pages, 16, hd).to(dtype), torch.arange(pages, dtype=torch.int32, device="cuda").repeat(batch, 1).contiguous()


def shared_attention64(q, k, v, n):
    out = torch.empty(q.shape, dtype=torch.float64, device="cuda")
    group = q.shape[1] // k.shape[0]
    for h in range(k.shape[0]):
        kh, vh = (x[h].reshape(-1, q.shape[2])[:n].double() for x in (k, v))
        of = slice(h * group, (h + 1) * group)
        out[:, of] = torch.softmax(q[:, of].double() @ kh.T * q.shape[2] ** -0.5, dim=-1) @ vh
    return out


def nearest_additions(n):
    """What n additions in turn, each rounded to nearest, are off relative to their sum of positive terms: roundings of a spread of 2^-24 / sqrt(3)
    at most, independent of one another; eight deviations."""
    return 8 / 3 ** 0.5 * n ** 0.5 * 2.0 ** -24


# a tile's own products and their sum, what warps and CTAs add, the quotient
TILE_AND_JOIN = 8 * 2.0 ** -23 + 24 * 2.0 ** -24


@pytest.mark.parametrize("hd,nq,nkv,batch,n,keys", [(32, 8, 8, 64, 40000, 16), (64, 8, 8, 64, 20000, 16), (128, 8, 8, 48, 20000, 8), (64, 8, 1, 500, 20000, 16)])
def test_fp32_attention_adds_long_stretches_in_fp32(lib, hd, nq, nkv, batch, n, keys):
    """Hundreds of tiles a warp, all weights 1 (so their sum is exact), values about 1: errors that all have one sign would show."""
    g = gen(hd)
    k, v, table = shared_pages(g, batch, nkv, n, hd, FP32, lambda *s: 1 + 0.2 * randn(g, *s))
    q = torch.zeros(batch, nq, hd, device="cuda")
    got = lib.hsd_paged_attention(q, k, v, table, ints([n] * batch)).double()
    want = shared_attention64(q, k, v, n)
    tiles = batch * nkv * n / keys / 1184 + 1
    assert tiles > 300
    off = float(((got - want).abs() / want).max())
    assert off <= TILE_AND_JOIN + nearest_additions(tiles), off


@pytest.mark.parametrize("hd,nq,keys", [(128, 8, 16), (64, 8, 32), (128, 72, 16)])
def test_bf16_attention_adds_long_stretches_in_fp32(lib, hd, nq, keys):
    """Means of 1 and its neighbour lie about their middle, where a small loss rounds down what should be rounded up."""
    g, nkv, batch, n = gen(hd + nq), 8, 64, 40000
    k, v, table = shared_pages(g, batch, nkv, n, hd, BF16, lambda *s: 1 + 2.0 ** -7 * torch.randint(0, 2, s, generator=g, device="cuda"))
    q = randn(g, batch, nq, hd, dtype=BF16, std=0.3)
    got = lib.hsd_paged_attention(q, k, v, table, ints([n] * batch)).double()
    want = shared_attention64(q, k, v, n)
    # a weight's error counts by the values' difference, 2^-7, alone; its sum: two additions for every 16 keys, in each of four lanes
    tiles = batch * nkv * n / keys / 1184 + 1
    bound = TILE_AND_JOIN + nearest_additions(tiles) + nearest_additions(tiles * keys / 8) / 2 + 2.0 ** -7 * 2.0 ** -18
    assert int((want > 1 + 2.0 ** -8 + 2 * bound).sum()) > 100
    assert bool(((got - want).abs() <= 2.0 ** -8 + bound * want).all()), float(((got - want).abs() - 2.0 ** -8).max())


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_attention_of_one_key_is_its_value(lib, dtype, hd):
    g = gen(hd + 1)
    k, v, table = cache(g, 40, 2, hd, 16, 1, dtype)
    v[0, table[3, 0], 0, 5], v[1, table[4, 0], 0, 6] = torch.finfo(dtype).max, torch.finfo(dtype).min
    got = lib.hsd_paged_attention(randn(g, 40, 6, hd, dtype=dtype, std=2.0), k, v, table, ints([1] * 40))
    want = v[:, table[:, 0].long(), 0].transpose(0, 1)                       # [batch, nkv, hd]
    assert torch.equal(got.view(40, 2, 3, hd), want[:, :, None].expand(40, 2, 3, hd))


def test_fp32_attention_takes_the_largest_queries(lib):
    """A query whose high part would be rounded to infinity, with keys small enough for finite scores."""
    g = gen(21)
    k, v, table = cache(g, 1, 1, 64, 16, 1, FP32)
    k *= 1e-38
    q = torch.zeros(1, 2, 64, device="cuda")
    q[0, 0, 7], q[0, 1, 9] = torch.finfo(FP32).max, torch.finfo(FP32).min
    got = lib.hsd_paged_attention(q, k, v, table, ints([12]))
    want, size, most = attention64(q, k, v, table.cpu(), [12], 0.125)
    # as in check_attention(); and factors are multiples of 2^-136, what TF32 holds below 2^-126: a key's two lower parts lose less than that
    # each, which counts 2^128 times 0.125 in a score
    weight = (64 + 4) * 2.0 ** -23 * most + 2.0 ** -21 + 66 * 2.0 ** -24 + 0.125 * 2.0 ** 128 * 2 * 2.0 ** -136
    assert bool(((got.double().cpu() - want).abs() <= 2.0 ** -24 * want.abs() + 2 * weight * size).all())


@pytest.mark.parametrize("nq", [8, 16])
def test_bf16_attention_weights_have_24_bits(lib, nq):
    """Sixteen keys, one of score 0, the others of one score whose weight the first 16 bits miss by 2e-6 and more.  Scores are exact (one product
    each).  A weight is off by 2^-22 (its exponential) and 2^-23 (the exponent, below 1), which counts by its share of the values' differences, a
    quarter at most; the tile's products 4 * 2^-23, the weights' sum and the quotient six roundings."""
    def missed(w):
        w = w.to(FP32)
        high = w.to(BF16).to(FP32)
        return ((w - high - (w - high).to(BF16).to(FP32)) / w).double()

    scores = -torch.arange(1, 180, device="cuda", dtype=torch.float64) / 256
    w = scores.exp()
    lo, hi = missed(w * (1 - 4e-7)), missed(w * (1 + 4e-7))
    safe = torch.where(lo.sign() == hi.sign(), torch.minimum(lo.abs(), hi.abs()), torch.zeros_like(lo))
    best = int(safe.argmax())
    assert float(safe[best]) > 2e-6
    g, batch, hd = gen(nq), 256, 128
    k, v, table = cache(g, batch, 1, hd, 16, 1, BF16)
    v.copy_(1 + torch.rand(v.shape, generator=g, device="cuda"))
    k.zero_()
    k[:, :, 1:, 0] = scores[best].to(BF16)
    assert float(k[0, 0, 1, 0]) == float(scores[best])
    q = torch.zeros(batch, nq, hd, dtype=BF16, device="cuda")
    q[:, :, 0] = 1
    got = lib.hsd_paged_attention(q, k, v, table, ints([16] * batch), 1.0).double()
    share = torch.cat((torch.ones(1, dtype=torch.float64, device="cuda"), w[best].expand(15)))
    share /= share.sum()
    want = (v[0, table[:, 0].long()].double() * share[:, None]).sum(dim=1)[:, None].expand(batch, nq, hd)
    off = (got - want).abs()
    bound = 2.0 ** -8 + (2.0 ** -22 + 2.0 ** -23) / 4 + (4 * 2.0 ** -23 + 6 * 2.0 ** -24) * want          # want lies in [1, 2]
    assert bool((off <= bound).all()), (float((off - 2.0 ** -8).max()), int((off > bound).sum()))


# ------------------------------------------------------------------------------------------------ append
def append64(qkv, table, before, rope, starts, nkv, pool_shape):
    """Rows' rotated queries and, by (row): (page, token, keys, values), in 64 bits; rows that are skipped are missing."""
    rows, heads, hd = qkv.shape
    nq, (n_pages, page) = heads - 2 * nkv, pool_shape
    x, t = qkv.double().cpu(), rope.double().cpu()
    found = {}
    for b, len0 in enumerate(before):
        for r in range(starts[b], min(starts[b + 1], rows)):
            p = len0 + r - starts[b]
            if len0 < 0 or p >= t.shape[0] or p >= table.shape[1] * page or not 0 <= int(table[b, p // page]) < n_pages:
                continue
            lo, hi = x[r, :nq + nkv, :hd // 2], x[r, :nq + nkv, hd // 2:]
            a, c = t[p, 0] * lo, t[p, 1] * hi
            d, e = t[p, 0] * hi, t[p, 1] * lo
            y, size = torch.cat((a - c, d + e), dim=1), torch.cat((a.abs() + c.abs(), d.abs() + e.abs()), dim=1)
            found[r] = (int(table[b, p // page]), p % page, y[:nq], y[nq:], x[r, nq + nkv:], size)
    return found


def check_append(lib, qkv, k, v, table, before, rope, starts=None, nq=None):
    nkv, n_pages, page, hd = k.shape
    q_out = torch.full((qkv.shape[0], qkv.shape[1] - 2 * nkv, hd), 7.0, dtype=k.dtype, device="cuda")
    k0, v0 = k.clone(), v.clone()
    edges = list(range(len(before) + 1)) if starts is None else starts
    found = append64(qkv, table.cpu(), before, rope, edges, nkv, (n_pages, page))
    got = lib.hsd_kv_append(qkv, k, v, table, ints(before), rope, None if starts is None else ints(starts), q_out)
    assert got is q_out
    touched = torch.zeros(n_pages, page, dtype=torch.bool)
    step = HALF_STEP[k.dtype]
    kc, vc, qc = k.cpu(), v.cpu(), q_out.cpu()
    for r, (pg, t, qy, ky, vx, size) in found.items():
        touched[pg, t] = True
        for out, want, s in ((qc[r], qy, size[:qy.shape[0]]), (kc[:, pg, t], ky, size[qy.shape[0]:])):
            assert bool(((out.double() - want).abs() <= step * want.abs() + 2 ** -22 * s).all())
        assert torch.equal(vc[:, pg, t], vx.to(FP32).to(k.dtype))
    left = torch.tensor([r for r in range(qkv.shape[0]) if r not in found], dtype=torch.long, device="cuda")
    assert bool((q_out[left] == 7.0).all())                                  # skipped rows: as they were
    keep = ~touched.cuda()
    assert torch.equal(k[:, keep], k0[:, keep]) and torch.equal(v[:, keep], v0[:, keep])
    return found


@pytest.mark.parametrize("source", [BF16, FP32])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("hd,nq,nkv,page,order", [(32, 4, 2, 16, "head"), (64, 1, 1, 3, "token"), (128, 8, 2, 16, "token"), (64, 0, 3, 8, "head")])
def test_append_one_token_each(lib, source, dtype, hd, nq, nkv, page, order):
    g = gen(hd + nq)
    before = [0, 1, 15, 16, 31, -1, 40]
    k, v, table = cache(g, 7, nkv, hd, page, -(-41 // page), dtype, order)
    found = check_append(lib, randn(g, 7, nq + 2 * nkv, hd, dtype=source), k, v, table, before, lib.rope_table(64, hd))
    assert sorted(found) == [0, 1, 2, 3, 4, 6]


@pytest.mark.parametrize("rows", [1, 40, 2500])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_append_ragged_rows(lib, rows, dtype):
    g = gen(rows)
    batch = 70                                                              # more than two ballots of row starts
    cut = sorted(torch.randint(0, rows + 1, (batch - 1,), generator=torch.Generator().manual_seed(rows)).tolist())
    starts = [0] + cut + [rows]
    before = [(i * 37) % 50 for i in range(batch)]
    longest = max(b + starts[i + 1] - starts[i] for i, b in enumerate(before))
    k, v, table = cache(g, batch, 1, 32, 16, -(-longest // 16), dtype)
    assert len(check_append(lib, randn(g, rows, 4, 32), k, v, table, before, lib.rope_table(longest, 32), starts)) == rows


def test_append_skips_what_has_no_place(lib):
    g = gen(3)
    k, v, table = cache(g, 4, 1, 64, 16, 2, BF16)
    table[1, 1], table[2, 0] = -1, k.shape[1]
    # rows in front of the first start and behind the last; past the pages (28 + 6 > 32); bad pages; past the rope table
    found = check_append(lib, randn(g, 30, 3, 64), k, v, table, [28, 14, 0, 18], lib.rope_table(30, 64), [2, 8, 13, 16, 25])
    assert sorted(found) == [2, 3, 8, 9] + list(range(16, 25))


def test_append_rows_that_lie_apart_and_far_positions(lib):
    g = gen(4)
    wide = randn(g, 5, 8 * 64, dtype=BF16)
    qkv = wide[:, 64:64 + 6 * 64].unflatten(1, (6, 64))
    before = [100000, 65535, 65536, 131071, 7]
    k, v = randn(g, 2, 6, 16, 64, dtype=BF16), randn(g, 2, 6, 16, 64, dtype=BF16)
    table = torch.zeros(5, 8192, dtype=torch.int32, device="cuda")
    table += ints([0, 1, 2, 3, 4])[:, None]
    assert len(check_append(lib, qkv, k, v, table, before, lib.rope_table(131072, 64))) == 5


@pytest.mark.parametrize("rows,starts", [(30, [2, 8, 13, 16, 25]), (1300, [5, 8, 13, 16, 1290]), (4, None)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_append_gives_zeros_for_queries_of_skipped_rows(lib, dtype, rows, starts):
    g = gen(rows)
    k, v, table = cache(g, 4, 1, 64, 16, 2, dtype)
    table[1, 1], table[2, 0] = -1, k.shape[1]
    before, rope, qkv = [28, 14, 0, -1 if starts is None else 18], lib.rope_table(30, 64), randn(g, rows, 5, 64)
    edges = list(range(5)) if starts is None else starts
    found = append64(qkv, table.cpu(), before, rope, edges, 1, (k.shape[1], 16))
    skipped = [r for r in range(rows) if r not in found]
    assert found and skipped
    into = torch.full((rows, 3, 64), 7.0, dtype=dtype, device="cuda")
    lib.hsd_kv_append(qkv, k, v, table, ints(before), rope, None if starts is None else ints(starts), into)
    for _ in range(3):
        dirt = torch.full((rows, 3, 64), float("nan"), dtype=dtype, device="cuda")          # what the next tensor of this size is made of
        del dirt
        q = lib.hsd_kv_append(qkv, k, v, table, ints(before), rope, None if starts is None else ints(starts))
        assert bool((q[skipped] == 0).all()) and torch.equal(q[sorted(found)], into[sorted(found)])


@pytest.mark.parametrize("rows", [2501, 2502, 2503])
def test_append_of_rows_that_are_not_whole_fours(lib, rows):
    g = gen(rows)
    k, v, table = cache(g, 3, 1, 32, 16, 70, BF16)
    found = check_append(lib, randn(g, rows, 4, 32, dtype=BF16), k, v, table, [3, 0, 17], lib.rope_table(1100, 32), [0, 1000, 1903, rows])
    assert len(found) == rows


# ------------------------------------------------------------------------------------------------ 4-bit products
def check_w4(lib, A, codes, scales, **more):
    got = lib.hsd_gemm_w4(A, codes, scales, **more)
    K, groups = A.shape[1], scales.shape[1]
    c = torch.stack((codes & 15, codes >> 4), dim=-1).view(codes.shape[0], K).double() - 8
    w = c * scales.double().repeat_interleave(K // groups, dim=1)
    want, size = A.double() @ w.T, A.double().abs() @ w.abs().T
    # K / 16 steps of the tensor cores' adders, each of them cut off at 2^-23, the scaling and the sums of groups and warps
    bound = (K / 16 + groups + 32) * 2.0 ** -23 * size + 1e-37
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), float((off / bound).max())
    return got


def weights(g, N, K, group):
    codes = torch.randint(0, 256, (N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    return codes, (0.01 * (0.1 + torch.rand(N, K // group, generator=g, device="cuda"))).to(BF16)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("N,groups", [(1, 1), (17, 3), (100, 8), (1000, 33)])
def test_w4_products(lib, group, rows, N, groups):
    g = gen(N + rows)
    check_w4(lib, randn(g, rows, group * groups, dtype=BF16), *weights(g, N, group * groups, group))


@pytest.mark.parametrize("rows,N,K,group", [(1, 4096, 4096, 128), (9, 14336, 4096, 128), (3, 4096, 14336, 64), (32, 32000, 2048, 32), (64, 4096, 4096, 128), (5, 129, 16384, 32)])
def test_w4_products_of_layers(lib, rows, N, K, group):
    g = gen(N)
    A, (codes, scales) = randn(g, rows, K, dtype=BF16), weights(g, N, K, group)
    got = check_w4(lib, A, codes, scales)
    out = torch.empty(rows, N, device="cuda")
    assert lib.hsd_gemm_w4(A, codes, scales, out=out) is out and torch.equal(out, got)       # sums in a fixed order


def test_w4_packed_weights_near_the_bf16_product(lib):
    g = gen(1)
    W, A = randn(g, 200, 512, dtype=BF16, std=0.02), randn(g, 4, 512, dtype=BF16)
    codes, scales = lib.w4_pack(W, 64)
    got = check_w4(lib, A, codes, scales)
    # every weight is off by at most half of its group's scale
    bound = A.double().abs() @ (0.5001 * scales.double().repeat_interleave(64, dim=1)).T
    assert bool(((got.double() - A.double() @ W.double().T).abs() <= bound * (1 + 1e-5)).all())


def test_w4_keeps_what_is_not_finite_to_its_row(lib):
    g = gen(2)
    A, (codes, scales) = randn(g, 3, 256, dtype=BF16), weights(g, 40, 256, 64)
    want = lib.hsd_gemm_w4(A, codes, scales)
    A2, s2 = A.clone(), scales.clone()
    A2[1, 7], s2[5, 2] = float("nan"), float("inf")
    got = lib.hsd_gemm_w4(A2, codes, s2)
    rows, cols = [0, 2], [i for i in range(40) if i != 5]
    assert bool(got[1].isnan().all()) and not bool(got[rows][:, 5].isfinite().any())
    assert torch.equal(got[rows][:, cols], want[rows][:, cols])


@pytest.mark.parametrize("rows,N,K,group", [(8, 28673, 4096, 128), (2, 32001, 4096, 128), (5, 32001, 2048, 32), (3, 40001, 2048, 64), (8, 40001, 2112, 64), (1, 33001, 1312, 32)])
def test_w4_products_of_few_rows_and_large_matrices(lib, rows, N, K, group):
    """Past the matrices whose few rows take one launch; groups that are not whole eights of a row."""
    g = gen(N)
    A, (codes, scales) = randn(g, rows, K, dtype=BF16), weights(g, N, K, group)
    got = check_w4(lib, A, codes, scales)
    assert torch.equal(lib.hsd_gemm_w4(A, codes, scales), got)


# ------------------------------------------------------------------------------------------------ log probabilities
def check_logprobs(lib, logits, tokens, top):
    lp, entropy, ranks, ids, top_lp = lib.hsd_token_logprobs(logits, tokens, top)
    V = logits.shape[-1]
    x, tok = logits.reshape(-1, V).double(), tokens.reshape(-1).long()
    d = x - x.amax(dim=1, keepdim=True)       # (x less log sum exp would lose the sum's logarithm beside a maximum of 1e38)
    want = d - d.exp().sum(dim=1, keepdim=True).log()
    p = want.exp()
    h = -torch.where(p > 0, p * want, torch.zeros_like(p)).sum(dim=1)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    given = (tok >= 0) & (tok < V)
    at = tok.clamp(0, V - 1)[:, None]
    # S: a thread adds up to V / 128 + 64 terms, an exponential is off by 2^-22 and by 2^-23 of its argument (at most 24 on average);
    # T has the same terms times their arguments
    sums = (V / 128 + 64) * 2.0 ** -24 + 2.0 ** -22 + 24 * 2.0 ** -23
    lp, entropy, ranks, ids, top_lp = lp.reshape(-1), entropy.reshape(-1), ranks.reshape(-1), ids.reshape(len(x), top), top_lp.reshape(len(x), top)

    def near(got, ref, bound):
        same = (got.double() == ref) | (got == ref.float())              # the latter: what passes fp32's range is its infinity
        assert bool((same | ((got.double() - ref).abs() <= bound)).all()), float((got.double() - ref).abs().max())

    ref = want.gather(1, at)[:, 0]
    near(lp[given], ref[given], (sums + 2.0 ** -22 * ref.abs())[given])
    assert bool(lp[~given].isnan().all()) and bool((ranks[~given] == -1).all())
    near(entropy, h, sums * (2 + 2 * h))
    place = torch.empty_like(order).scatter_(1, order, torch.arange(V, device="cuda").expand_as(order).contiguous())
    assert torch.equal(ranks[given].long(), place.gather(1, at)[:, 0][given])
    assert torch.equal(ids.long(), order[:, :top])
    ref = want.gather(1, order[:, :top])
    near(top_lp, ref, sums + 2.0 ** -22 * ref.abs())


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", [1, 2, 7, 33, 512, 1000, 2049, 4096, 4097, 32000, 32001, 131072, 150001])
@pytest.mark.parametrize("rows", [1, 3, 40])
def test_logprobs_of_any_vocabulary(lib, dtype, V, rows):
    g = gen(V + rows)
    tokens = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    for top in sorted({0, 1, min(5, V), min(32, V)}):
        check_logprobs(lib, randn(g, rows, V, std=3.0, dtype=dtype), tokens, top)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", [9, 100, 257, 1461, 2048])
def test_logprobs_of_many_short_rows(lib, dtype, V):
    g = gen(V)
    x = randn(g, 700, V, std=3.0, dtype=dtype)
    x[::7] = x[::7].round()                       # ties
    x[3::9, V // 2:] = -float("inf")
    x[5::50] = 2.0
    tokens = torch.randint(0, V, (700,), generator=g, device="cuda", dtype=torch.int32)
    for top in (0, 1, 5, 8):
        check_logprobs(lib, x, tokens, top)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", [500, 32000, 70001])
def test_logprobs_of_ties(lib, dtype, V):
    """Rows with more equal logits than candidates fit: all equal, few values, a mask that leaves three tokens, ties at the far end."""
    g = gen(V)
    x = torch.zeros(8, V, device="cuda")
    x[1] = torch.randint(0, 3, (V,), generator=g, device="cuda").float()
    x[2] = -float("inf")
    x[2, [7, V // 2, V - 1]] = torch.tensor([1.0, 2.0, 1.0], device="cuda")
    x[3, -9:] = 2.0
    x[4] = torch.arange(V, device="cuda") // 64
    x[5] = -(torch.arange(V, device="cuda") // 64).float()
    x[6, ::2] = -0.0
    x[7] = torch.finfo(dtype).min
    x[7, V - 2] = 0.0
    tokens = ints([0, V - 1, 7, V - 3, V // 2, V // 3, 3, V - 1])
    for top in (0, 1, 5, 20, 32):
        check_logprobs(lib, x.to(dtype), tokens, top)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,V", [(300, 4099), (300, 32001), (300, 70001), (100, 262147), (1, 524291)])
def test_logprobs_of_many_and_of_long_rows(lib, dtype, rows, V):
    """A CTA a row, and CTAs of 512 threads alone and in clusters; odd rows lie off 16-byte boundaries."""
    g = gen(V)
    x = randn(g, rows, V, std=3.0, dtype=dtype)
    if rows > 1:
        x[1::6] = x[1::6].round()                                            # ties
        x[2::6, V // 3:] = -float("inf")
        x[3::6] = 2.0                                                        # more equals than candidates
        x[4::12, : V - 7] = torch.finfo(dtype).min
        x[5::12] = -float("inf")
        x[5::12, ::V // 3] = 1.0                                             # three tokens
    tokens = torch.randint(0, V, (rows,), generator=g, device="cuda", dtype=torch.int32)
    for top in (0, 5, 32):
        check_logprobs(lib, x, tokens, top)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", [300, 32000])
def test_logprobs_of_extreme_rows(lib, dtype, V):
    g = gen(V + 1)
    big = torch.finfo(dtype).max
    x = randn(g, 6, V, std=1.0)
    x[0] += 3e4                                   # far from 0
    x[1] = torch.where(torch.arange(V, device="cuda") % 2 == 0, big, -big).float()
    x[2] = -big
    x[3, 11] = 1000.0                             # one token has it all
    x[4] *= 100
    x[5] = -float("inf")
    x[5, V - 1] = -big
    check_logprobs(lib, x.to(dtype), ints([1, 1, V - 1, 11, 5, V - 1]), 5)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("V", [300, 32000])
def test_logprobs_of_rows_without_a_distribution(lib, dtype, V):
    g = gen(V + 2)
    x = randn(g, 5, V, dtype=dtype)
    x[0, 5], x[1, V - 1], x[2], x[3, 0] = float("nan"), float("inf"), -float("inf"), -float("inf")
    lp, entropy, ranks, ids, top_lp = lib.hsd_token_logprobs(x, ints([4, 4, 4, 0, -1]), 3)
    assert bool(lp[:2].isnan().all()) and bool(entropy[:2].isnan().all()) and ranks[:2].tolist() == [-1, -1]
    assert bool((ids[:2] == -1).all()) and bool(top_lp[:2].isnan().all())
    assert float(lp[2]) == -math.inf and float(entropy[2]) == 0 and int(ranks[2]) == 4 and ids[2].tolist() == [0, 1, 2] and bool((top_lp[2] == -math.inf).all())
    assert float(lp[3]) == -math.inf and int(ranks[3]) == V - 1
    assert math.isnan(float(lp[4])) and int(ranks[4]) == -1 and bool(top_lp[4].isfinite().all())


def test_logprobs_shapes_alignment_and_padding(lib):
    g = gen(12)
    base = randn(g, 2 * 3 * 1003 + 1, dtype=BF16)
    x = base[1:].view(2, 3, 1003)                 # no row on a 16-byte boundary
    tokens = ints([[1, 2, -1], [1002, 1003, -1]])  # as hsd_verify_level pads, and one past the end
    check_logprobs(lib, x, tokens, 7)
    lp, entropy, ranks, ids, top_lp = lib.hsd_token_logprobs(x, tokens, 7)
    assert lp.shape == entropy.shape == ranks.shape == (2, 3) and ids.shape == top_lp.shape == (2, 3, 7)
    with pytest.raises(ValueError):
        lib.hsd_token_logprobs(x, tokens[0], 7)
    with pytest.raises(lib.HsdError):
        lib.hsd_token_logprobs(x, tokens.long(), 7)
    with pytest.raises(lib.HsdError, match="invalid argument"):
        lib.hsd_token_logprobs(x, tokens, 33)


def test_the_binding_refuses_shapes_and_types(lib):
    g = gen(13)
    k, v, table = cache(g, 2, 2, 64, 16, 4, BF16)
    q, lens, rope, qkv = randn(g, 2, 4, 64, dtype=BF16), ints([3, 4]), lib.rope_table(64, 64), randn(g, 2, 8, 64)
    for wrong in (dict(q=q[:1]), dict(lens=lens[:1]), dict(v=v[:, :2]), dict(q=q[..., :32].contiguous()), dict(v=v.permute(0, 2, 1, 3))):
        d = dict(q=q, k=k, v=v, table=table, lens=lens)
        d.update(wrong)
        with pytest.raises(ValueError):
            lib.hsd_paged_attention(*d.values())
    for wrong in (dict(q=q.float()), dict(lens=lens.long()), dict(k=k.half(), v=v.half()), dict(k=k.transpose(2, 3), v=v.transpose(2, 3)), dict(table=table.T.contiguous().T),
                  dict(q=randn(g, 2, 3, 64, dtype=BF16))):
        d = dict(q=q, k=k, v=v, table=table, lens=lens)
        d.update(wrong)
        with pytest.raises((lib.HsdError, ValueError)):
            lib.hsd_paged_attention(*d.values())
    for wrong in (dict(qkv=qkv[:, :3].contiguous()), dict(rope=rope[:, :, :16].contiguous()), dict(starts=ints([0, 1]))):
        d = dict(qkv=qkv, k=k, v=v, table=table, lens=lens, rope=rope, starts=None)
        d.update(wrong)
        with pytest.raises(ValueError):
            lib.hsd_kv_append(*d.values())
    with pytest.raises(lib.HsdError, match="workspace too small"):
        lib.hsd_paged_attention(q, k, v, table, lens, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    codes, scales = weights(g, 8, 128, 64)
    A = randn(g, 2, 128, dtype=BF16)
    for a, c, s in ((A.float(), codes, scales), (A, codes, scales.float()), (A.T.contiguous().T, codes, scales), (randn(g, 65, 128, dtype=BF16), codes, scales)):
        with pytest.raises(lib.HsdError):
            lib.hsd_gemm_w4(a, c, s)
    for c, s in ((codes[:, :32].contiguous(), scales), (codes, scales[:4])):
        with pytest.raises(ValueError):
            lib.hsd_gemm_w4(A, c, s)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_logprobs_of_the_largest_vocabulary(lib, dtype):
    """Ids up to 2^31 - 257, whose steps of a thread's next pieces would pass 2^31."""
    V = (1 << 31) - 256
    x = torch.zeros(1, V, dtype=dtype, device="cuda")
    x[0, V - 5] = 2.0
    ref = -math.log(V - 1 + math.exp(2.0))
    for t, rank, logit in ((5, 6, 0.0), (V - 20000, V - 19999, 0.0), (V - 300, V - 299, 0.0), (V - 5, 0, 2.0), (V - 1, V - 1, 0.0)):
        lp, _, ranks, ids, _ = lib.hsd_token_logprobs(x, ints([t]), 3)
        assert int(ranks) == rank and ids.tolist() == [[V - 5, 0, 1]]
        assert abs(float(lp) - logit - ref) < 2e-5                          # 2^31 / (8 * 512) terms a thread, each rounded: 2^19 * 2^-24 at the very most is 0.03


# ------------------------------------------------------------------------------------------------ together
def test_a_drafter_of_ones_own(lib):
    """Two layers with 4-bit projections decode three sequences of different lengths over a paged cache: prompts in one ragged append,
    then steps of one token; every step's logits against a plain forward in 64 bits with the same rounding points, its draws by hsd_draft_sample
    and what they were worth by hsd_token_logprobs, a verification of the drafts at the end."""
    g = gen(77)
    d, nq, nkv, hd, ff, V, page, layers, steps = 256, 4, 2, 64, 512, 1000, 16, 2, 5
    prompts = [37, 1, 20]
    B = len(prompts)

    def pack(n, k):
        codes, scales = lib.w4_pack(randn(g, n, k, std=0.06), 64)
        c = torch.stack((codes & 15, codes >> 4), dim=-1).view(n, k).double() - 8
        return codes, scales, (c * scales.double().repeat_interleave(64, dim=1)).cpu()

    W = [dict(qkv=pack((nq + 2 * nkv) * hd, d), o=pack(d, nq * hd), up=pack(ff, d), down=pack(d, ff)) for _ in range(layers)]
    head, embed = pack(V, d), randn(g, V, d, dtype=BF16)
    rope = lib.rope_table(64, hd)
    k_pools, v_pools, tables = zip(*(cache(g, B, nkv, hd, page, 4, BF16, spare=2) for _ in range(layers)))

    def norm(x):
        return x * torch.rsqrt(x.square().mean(dim=-1, keepdim=True) + 1e-5)

    def product(x, w):                                                      # in pieces: at most 64 rows a call
        x = x.to(BF16).contiguous()
        return torch.cat([lib.hsd_gemm_w4(p.contiguous(), w[0], w[1]) for p in x.split(64)])

    def attend(l, qkv, lens, starts, i):
        """Rows' attention: each row as a call of its own length, so that prompts take the decoding path too."""
        q = lib.hsd_kv_append(qkv.view(-1, nq + 2 * nkv, hd), k_pools[l], v_pools[l], tables[l], ints(lens), rope, None if starts is None else ints(starts))
        if starts is None:
            return lib.hsd_paged_attention(q, k_pools[l], v_pools[l], tables[l], ints([n + 1 for n in lens]))
        seq = [b for b in range(B) for _ in range(starts[b + 1] - starts[b])]
        upto = [lens[b] + r + 1 for b in range(B) for r in range(starts[b + 1] - starts[b])]
        return lib.hsd_paged_attention(q, k_pools[l], v_pools[l], tables[l][torch.tensor(seq)].contiguous(), ints(upto))

    def forward(tokens, lens, starts=None):
        x = embed[tokens].float()
        for l in range(layers):
            a = attend(l, product(norm(x), W[l]["qkv"]), lens, starts, l)
            x = x + product(a.reshape(-1, nq * hd), W[l]["o"])
            x = x + product(torch.nn.functional.gelu(product(norm(x), W[l]["up"])), W[l]["down"])
        return product(norm(x), head)

    def plain(tokens):
        """The last position's logits of one sequence, in 64 bits but for the rounding points."""
        bf = lambda t: t.float().to(BF16).double()
        x = embed.cpu()[tokens].double()
        n = len(tokens)
        t = rope.cpu().double()[:n]
        for l in range(layers):
            qkv = (bf(norm(x)) @ W[l]["qkv"][2].T).view(n, nq + 2 * nkv, hd)
            lo, hi = qkv[:, :nq + nkv, :hd // 2], qkv[:, :nq + nkv, hd // 2:]
            c, s = t[:, 0, None], t[:, 1, None]
            qk = bf(torch.cat((lo * c - hi * s, hi * c + lo * s), dim=-1))
            q, k, v = qk[:, :nq], qk[:, nq:], bf(qkv[:, nq + nkv:])
            k, v = (z.repeat_interleave(nq // nkv, dim=1) for z in (k, v))
            w = torch.einsum("ihd,jhd->hij", q, k) * hd ** -0.5
            w = torch.softmax(w.masked_fill(torch.ones(n, n).triu(1).bool(), -math.inf), dim=-1)
            x = x + bf(torch.einsum("hij,jhd->ihd", w, v).reshape(n, nq * hd)) @ W[l]["o"][2].T
            x = x + bf(torch.nn.functional.gelu(bf(norm(x)) @ W[l]["up"][2].T)) @ W[l]["down"][2].T
        return bf(norm(x[-1])) @ head[2].T

    text = [torch.randint(0, V, (n,), generator=torch.Generator().manual_seed(n)).tolist() for n in prompts]
    starts = [0, 37, 38, 58]
    logits = forward(torch.tensor(sum(text, []), device="cuda"), [0] * B, starts)[torch.tensor([36, 37, 57], device="cuda")]
    rows, drafts = [], []
    for step in range(steps):
        for b in range(B):                                                  # the bf16 forwards' own bound: a few flips of a rounding
            assert float((logits[b].double().cpu() - plain(text[b])).abs().max()) < 2e-2
        tokens = lib.hsd_draft_sample(logits.view(B, 1, V), 5, step)[:, 0]
        check_logprobs(lib, logits, tokens, 8)
        rows.append(logits.clone())
        drafts.append(tokens.clone())
        lens = [len(t) for t in text]
        for b in range(B):
            text[b].append(int(tokens[b]))
        logits = forward(tokens.long(), lens)
    q = torch.stack(rows, dim=1).contiguous()
    out, n = lib.hsd_verify_level(1, torch.cat((q, logits[:, None]), dim=1).contiguous(), q, torch.stack(drafts, dim=1).contiguous(), 5, 0)
    assert n.tolist() == [steps] * B                                        # verified by itself: everything is accepted
    lp = lib.hsd_token_logprobs(torch.cat((q, logits[:, None]), dim=1).contiguous(), out)[0]
    assert bool((lp <= 0).all()) and bool(lp.isfinite().all())


def _step(lib, s):
    """A decoding step's four calls on the tensors of `s`, none of which the calls keep."""
    q = lib.hsd_kv_append(s["qkv"], s["k"], s["v"], s["table"], s["lens"], s["rope"])
    a = lib.hsd_paged_attention(q, s["k"], s["v"], s["table"], s["upto"])
    logits = lib.hsd_gemm_w4(a.view(a.shape[0], -1), s["codes"], s["scales"])
    return (a, logits) + lib.hsd_token_logprobs(logits, s["tokens"], 5)


def _step_inputs(lib, seed, batch, N):
    g = gen(seed)
    k, v, table = cache(g, batch, 2, 64, 16, 30, BF16)
    codes, scales = weights(g, N, 256, 64)
    lens = torch.randint(0, 460, (batch,), generator=g, device="cuda", dtype=torch.int32)
    return dict(qkv=randn(g, batch, 8, 64), k=k, v=v, table=table, lens=lens, upto=lens + 1, rope=lib.rope_table(480, 64), codes=codes, scales=scales,
                tokens=torch.randint(0, N, (batch,), generator=g, device="cuda", dtype=torch.int32))


@pytest.mark.parametrize("batch,N", [(1, 9000), (12, 2500), (40, 70000)])
def test_captured_steps_follow_their_inputs(lib, batch, N):
    s = _step_inputs(lib, batch, batch, N)
    _step(lib, s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(lib, s)
    for seed in (1, 2, 3):
        other = _step_inputs(lib, seed, batch, N)
        for name, t in other.items():
            s[name].copy_(t)
        graph.replay()
        graph.replay()
        want = _step(lib, other)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert torch.equal(s["k"], other["k"]) and torch.equal(s["v"], other["v"])


def test_steps_on_two_streams_at_once(lib):
    sides = [_step_inputs(lib, 5, 9, 40000), _step_inputs(lib, 6, 33, 9000)]
    want = [_step(lib, s) for s in sides]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in sides], [[], []]
    for _ in range(20):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(_step(lib, sides[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for out in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(out, want[i]))
