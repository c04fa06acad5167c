"""The operators of a caller's own drafter refuse what they cannot take, before any CUDA call; packing and tables are plain torch."""
import ctypes

import pytest
import torch

from paper_2510_19705_b200 import binding

P = 1 << 20                    # an address that is never read: the refusals come first


def pool(**k):
    d = dict(k=P, v=P, dtype=1, n_pages=4, page_size=16, head_stride=4 * 16 * 64, page_stride=16 * 64, token_stride=64)
    d.update(k)
    return binding._KvPool(*(d[n] for n, _ in binding._KvPool._fields_))


def append(p=None, **k):
    d = dict(qkv=P, dtype=0, rows=2, row_stride=8 * 64, nq=4, nkv=2, hd=64, starts=None, lens=P, batch=2, table=P, pages=3, rope=P, positions=64)
    q_out = k.pop("q_out", P)
    d.update(k)
    return binding.library().hsd_kv_append(*d.values(), ctypes.byref(p or pool()), q_out, None)


def attention(p=None, **k):
    d = dict(q=P, batch=2, nq=4, nkv=2, hd=64)
    e = dict(table=P, pages=3, lens=P, scale=0.125, ws=P, ws_bytes=1 << 30, out=P)
    for name, v in k.items():
        (d if name in d else e)[name] = v
    return binding.library().hsd_paged_attention(*d.values(), ctypes.byref(p or pool()), *e.values(), None)


@pytest.mark.parametrize("bad", [dict(qkv=None), dict(rows=0), dict(rows=3), dict(row_stride=8 * 64 - 16), dict(row_stride=8 * 64 + 1), dict(nq=-1), dict(nkv=0),
                                 dict(lens=None), dict(batch=0), dict(table=None), dict(pages=0), dict(rope=None), dict(positions=0), dict(qkv=P + 4),
                                 dict(rope=P + 4), dict(q_out=None), dict(q_out=P + 2), dict(dtype=2)])
def test_append_refuses_arguments(bad):
    assert append(**bad) == -1


@pytest.mark.parametrize("call", [append, attention])
def test_pools_are_checked(call):
    for bad in (dict(k=None), dict(v=None), dict(k=P + 8), dict(dtype=3), dict(n_pages=0), dict(page_size=0), dict(head_stride=-64), dict(page_stride=1), dict(token_stride=4)):
        assert call(pool(**bad)) == -1, bad
    assert call(hd=48) == -6 and call(pool(page_size=1 << 30), pages=3) == -8


def test_sizes_past_the_limits():
    assert append(nq=65536, row_stride=1 << 30) == -8
    assert attention(batch=4097) == -8
    assert attention(nq=131072) == -8
    assert attention(pool(page_size=1 << 20), batch=4096, pages=3) == -8
    lib = binding.library()
    assert lib.hsd_gemm_w4(P, 1, (1 << 27) + 128, P, P, 8, 128, P, P, 1 << 40, None) == -8
    assert lib.hsd_token_logprobs(P, 0, 1, (1 << 31) - 1, P, 0, P, P, P, None, None, None) == -8


@pytest.mark.parametrize("bad", [dict(q=None), dict(batch=0), dict(nq=0), dict(nkv=3), dict(table=None), dict(pages=0), dict(lens=None), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(ws=None), dict(ws=P + 4), dict(out=None), dict(out=P + 2), dict(q=P + 8)])
def test_attention_refuses_arguments(bad):
    assert attention(**bad) == -1


def test_attention_workspace():
    size = binding.hsd_paged_attention_workspace_bytes
    assert size(4, 3, 64) == size(0, 1, 64) == size(4, 0, 64) == size(4, 2, 48) == 0
    assert attention(ws_bytes=size(4, 2, 64) - 1) == -2


@pytest.mark.parametrize("bad", [(None, 1, 128, P, P, 8, 128, P), (P, 0, 128, P, P, 8, 128, P), (P, 65, 128, P, P, 8, 128, P), (P, 1, 96, P, P, 8, 128, P),
                                 (P, 1, 0, P, P, 8, 128, P), (P, 1, 128, None, P, 8, 128, P), (P, 1, 128, P, None, 8, 128, P), (P, 1, 128, P, P, 0, 128, P),
                                 (P, 1, 128, P, P, 8, 16, P), (P, 1, 128, P, P, 8, 0, P), (P, 1, 128, P, P, 8, 128, None), (P + 2, 1, 128, P, P, 8, 128, P),
                                 (P, 1, 128, P + 1, P, 8, 128, P), (P, 1, 128, P, P + 1, 8, 128, P), (P, 1, 128, P, P, 8, 128, P + 2)])
def test_gemm_w4_refuses_arguments(bad):
    assert binding.library().hsd_gemm_w4(*bad, P, 1 << 40, None) == -1


def test_gemm_w4_workspace():
    size, call = binding.hsd_gemm_w4_workspace_bytes, binding.library().hsd_gemm_w4
    assert size(0, 8, 128, 128) == size(65, 8, 128, 128) == size(1, 0, 128, 128) == size(1, 8, 96, 64) == size(1, 8, 128, 16) == 0
    assert call(P, 3, 128, P, P, 8, 128, P, P, size(3, 8, 128, 128) - 1, None) == -2
    assert call(P, 3, 128, P, P, 8, 128, P, None, 1 << 40, None) == -1 and call(P, 3, 128, P, P, 8, 128, P, P + 4, 1 << 40, None) == -1


@pytest.mark.parametrize("bad", [dict(logits=None), dict(dtype=2), dict(rows=0), dict(vocab=0), dict(tokens=None), dict(top=-1), dict(top=33), dict(vocab=8, top=9),
                                 dict(lp=None), dict(entropy=None), dict(ranks=None), dict(top=1, ids=None), dict(top=1, top_lp=None), dict(logits=P + 1)])
def test_token_logprobs_refuses_arguments(bad):
    d = dict(logits=P, dtype=1, rows=2, vocab=64, tokens=P, top=0, lp=P, entropy=P, ranks=P, ids=P, top_lp=P)
    d.update(bad)
    assert binding.library().hsd_token_logprobs(*d.values(), None) == -1


def test_the_binding_wants_cuda_tensors():
    f, b, i = torch.zeros(2, 8, 64), torch.zeros(2, 4, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32)
    calls = (lambda: binding.hsd_kv_append(f, b, b, i, i[:, 0], f), lambda: binding.hsd_paged_attention(f, b, b, i, i[:, 0]),
             lambda: binding.hsd_gemm_w4(b[0, 0], i, f), lambda: binding.hsd_token_logprobs(f, i, 4))
    for call in calls:
        with pytest.raises(binding.HsdError, match="CUDA tensor"):
            call()
    with pytest.raises(ValueError):
        binding.hsd_kv_append(f[0], b, b, i, i[:, 0], f)
    with pytest.raises(TypeError):
        binding.hsd_gemm_w4(None, i, f)
    with pytest.raises(binding.HsdError, match="unsupported logits dtype"):
        binding.hsd_token_logprobs(f.double(), i, 4)


def unpack(codes, scales):
    c = torch.stack((codes & 15, codes >> 4), dim=-1).view(codes.shape[0], -1).double() - 8
    return c * scales.double().repeat_interleave(c.shape[1] // scales.shape[1], dim=1)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_packed_weights_are_the_nearest_codes(group, dtype):
    W = (torch.randn(5, 4 * group, generator=torch.Generator().manual_seed(group)) * 0.02).to(dtype)
    W[1, :group] = 0
    W[2, group] = 1.0
    codes, scales = binding.w4_pack(W, group)
    assert codes.dtype == torch.uint8 and codes.shape == (5, 2 * group) and scales.shape == (5, 4) and scales.dtype == torch.bfloat16
    # the scale is within 2^-8 of max / 7, so |w| < 7.03 scales, and the nearest code at most half a step away
    assert bool(((unpack(codes, scales) - W.double()).abs() <= 0.5001 * scales.double().repeat_interleave(group, dim=1)).all())
    assert bool((unpack(codes, scales)[1, :group] == 0).all())


def test_packing_marks_groups_that_are_not_finite_and_refuses_sizes():
    W = torch.ones(2, 64)
    W[0, 3], W[1, 40] = float("inf"), float("nan")
    codes, scales = binding.w4_pack(W, 32)
    assert torch.isnan(scales.float()).tolist() == [[True, False], [False, True]]
    for n, g in ((64, 48), (96, 64)):
        with pytest.raises(binding.HsdError):
            binding.w4_pack(torch.ones(1, n), g)


def test_rope_table():
    t = binding.rope_table(70000, 64, device="cpu")
    assert t.shape == (70000, 2, 32) and t.dtype == torch.float32
    a = 69999 * 10000.0 ** (-2 * 5 / 64)
    assert float(t[69999, 0, 5]) == pytest.approx(float(torch.tensor(a, dtype=torch.float64).cos()), abs=2 ** -24)
    assert float(t[69999, 1, 5]) == pytest.approx(float(torch.tensor(a, dtype=torch.float64).sin()), abs=2 ** -24)


def test_append_with_zeros_refuses_what_append_refuses():
    def call(**k):
        d = dict(qkv=P, dtype=0, rows=2, row_stride=8 * 64, nq=4, nkv=2, hd=64, starts=None, lens=P, batch=2, table=P, pages=3, rope=P, positions=64)
        d.update(k)
        return binding.library().hsd_kv_append_zeros(*d.values(), ctypes.byref(pool()), P, None)

    assert call(qkv=None) == call(rows=3) == call(rope=P + 4) == -1 and call(hd=48) == -6


def test_gemm_w4_refuses_rows_past_32_bits():
    """Tiles of 128 weight rows go up to 255 past the last: their numbers have to fit."""
    call = binding.library().hsd_gemm_w4
    for n in ((1 << 31) - 1, (1 << 31) - 255):
        for r, k, group in ((1, 32, 32), (9, 128, 128)):
            assert call(P, r, k, P, P, n, group, P, P, 1 << 40, None) == -8


@pytest.mark.parametrize("scale", [3e38, -3e38, 2.4e38])
def test_attention_refuses_a_scale_that_is_infinite_in_powers_of_two(scale):
    assert attention(scale=scale) == -1


def test_lists_of_words_have_to_be_aligned():
    for name in ("starts", "lens", "table"):
        assert append(**{name: P + 2}) == -1, name
    for name in ("lens", "table"):
        assert attention(**{name: P + 1}) == -1, name
    for name in ("tokens", "lp", "entropy", "ranks", "ids", "top_lp"):
        d = dict(logits=P, dtype=1, rows=2, vocab=64, tokens=P, top=1, lp=P, entropy=P, ranks=P, ids=P, top_lp=P)
        d[name] = P + 2
        assert binding.library().hsd_token_logprobs(*d.values(), None) == -1, name
