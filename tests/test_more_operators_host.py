"""The operators of a decoding step over continuations of one prompt refuse what they cannot take, before any CUDA call."""
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
    d = dict(qkv=P, dtype=0, rows=2, row_stride=8 * 64, nq=4, nkv=2, hd=64, q_gain=P, k_gain=P, gain_dtype=1, eps=1e-6, starts=None, lens=P, batch=2, table=P,
             pages=3, rope=P, positions=64)
    q_out = k.pop("q_out", P)
    d.update(k)
    return binding.library().hsd_kv_append_norm(*d.values(), ctypes.byref(p or pool()), 1, q_out, None)


def prefix(p=None, **k):
    d = dict(q=P, rows=2, nq=4, nkv=2, hd=64)
    e = dict(table=P, pages=3, lens=P, starts=None, batch=2, prefix=P, prefix_pages=2, prefix_len=P, scale=0.125, ws=P, ws_bytes=1 << 40, zeros=1, out=P)
    for name, v in k.items():
        (d if name in d else e)[name] = v
    return binding.library().hsd_prefix_attention(*d.values(), ctypes.byref(p or pool()), *e.values(), None)


def w8(**k):
    d = dict(A=P, a_dtype=1, a_scales=None, R=3, K=64, codes=P, scales=P, N=8, out=P, out_dtype=0, ws=P, ws_bytes=1 << 40)
    d.update(k)
    return binding.library().hsd_gemm_w8(*d.values(), None)


def quantize(**k):
    d = dict(x=P, dtype=1, rows=3, K=64, stride=64, codes=P, scales=P)
    d.update(k)
    return binding.library().hsd_quantize_rows(*d.values(), None)


@pytest.mark.parametrize("bad", [dict(qkv=None), dict(rows=0), dict(rows=3), dict(row_stride=8 * 64 - 16), dict(nq=-1), dict(nkv=0), dict(lens=None), dict(batch=0), dict(table=None),
                                 dict(pages=0), dict(rope=None), dict(positions=0), dict(qkv=P + 4), dict(rope=P + 4), dict(q_out=None), dict(dtype=2), dict(lens=P + 2),
                                 dict(q_gain=P + 8), dict(k_gain=P + 2), dict(gain_dtype=2), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf"))])
def test_append_norm_refuses_arguments(bad):
    assert append(**bad) == -1


@pytest.mark.parametrize("call", [append, prefix])
def test_pools_are_checked(call):
    for bad in (dict(k=None), dict(v=None), dict(k=P + 8), dict(dtype=3), dict(n_pages=0), dict(page_size=0), dict(head_stride=-64), dict(page_stride=1), dict(token_stride=4)):
        assert call(pool(**bad)) == -1, bad
    assert call(hd=48) == -6 and call(pool(page_size=1 << 30), pages=3) == -8


@pytest.mark.parametrize("bad", [dict(q=None), dict(rows=0), dict(rows=3), dict(batch=0), dict(nq=0), dict(nkv=3), dict(table=None), dict(pages=0), dict(lens=None), dict(prefix=None),
                                 dict(prefix_pages=0), dict(prefix_len=None), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(ws=None), dict(ws=P + 128),
                                 dict(out=None), dict(out=P + 2), dict(q=P + 8), dict(table=P + 2), dict(lens=P + 1), dict(starts=P + 2), dict(prefix=P + 2), dict(prefix_len=P + 3)])
def test_prefix_attention_refuses_arguments(bad):
    assert prefix(**bad) == -1


def test_prefix_attention_sizes_and_workspace():
    size = binding.hsd_prefix_attention_workspace_bytes
    assert size(0, 4, 2, 64) == size(2, 4, 3, 64) == size(2, 0, 1, 64) == size(2, 4, 2, 48) == size(1 << 20, 1 << 10, 8, 64) == 0
    assert prefix(ws_bytes=size(2, 4, 2, 64) - 1) == -2
    assert prefix(batch=4097, rows=4097) == -8 and prefix(nq=131072) == -8 and prefix(rows=1 << 25, starts=P) == -8
    assert prefix(pool(page_size=1 << 20), batch=4096, rows=4096, pages=2000) == -8                  # tiles past 2^31
    assert prefix(pool(page_size=1 << 20), prefix_pages=1 << 12) == -8


@pytest.mark.parametrize("bad", [dict(A=None), dict(a_dtype=3), dict(a_dtype=2), dict(a_scales=P), dict(R=0), dict(K=0), dict(K=24), dict(codes=None), dict(codes=P + 8), dict(scales=None),
                                 dict(scales=P + 2), dict(N=0), dict(out=None), dict(out=P + 2), dict(out_dtype=2), dict(out_dtype=1, out=P + 1), dict(ws=None), dict(ws=P + 16), dict(A=P + 1),
                                 dict(a_dtype=0, A=P + 2), dict(a_dtype=2, a_scales=P, A=P + 8), dict(a_dtype=2, a_scales=P + 2)])
def test_gemm_w8_refuses_arguments(bad):
    assert w8(**bad) == -1


def test_gemm_w8_sizes_and_workspace():
    size = binding.hsd_gemm_w8_workspace_bytes
    assert size(1, 0, 8, 64) == size(1, 3, 0, 64) == size(1, 3, 8, 24) == size(3, 3, 8, 64) == size(1, 3, 8, 1 << 17) == 0
    assert size(2, 1000, 8, 64) == 256 and size(1, 1000, 8, 64) >= 1000 * 68
    assert w8(ws_bytes=size(1, 3, 8, 64) - 1) == -2 and w8(a_dtype=2, a_scales=P, ws_bytes=255) == -2
    assert w8(K=1 << 17) == -8 and w8(N=(1 << 31) - 1) == -8 and w8(R=(1 << 31) - 1) == -8 and w8(R=1 << 22, N=1 << 24) == -8


@pytest.mark.parametrize("bad", [dict(x=None), dict(dtype=2), dict(rows=0), dict(K=0), dict(stride=63), dict(codes=None), dict(scales=None), dict(scales=P + 2), dict(x=P + 1),
                                 dict(dtype=0, x=P + 2)])
def test_quantize_rows_refuses_arguments(bad):
    assert quantize(**bad) == -1


def test_quantize_rows_sizes():
    assert quantize(K=(1 << 31) - 1, stride=1 << 31) == -8


def test_the_binding_wants_cuda_tensors_of_the_right_types():
    f, b, i = torch.zeros(2, 8, 64), torch.zeros(2, 4, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 3, dtype=torch.int32)
    calls = (lambda: binding.hsd_kv_append_norm(f, None, None, 1e-6, b, b, i, i[:, 0], f), lambda: binding.hsd_prefix_attention(f, b, b, i, i[:, 0], i[0], i[0, :1]),
             lambda: binding.hsd_gemm_w8(f[0], i, f), lambda: binding.hsd_quantize_rows(f[0]))
    for call in calls:
        with pytest.raises(binding.HsdError, match="CUDA tensor"):
            call()
    with pytest.raises(ValueError):
        binding.hsd_quantize_rows(f)
    with pytest.raises(TypeError):
        binding.hsd_gemm_w8(None, i, f)
    with pytest.raises(binding.HsdError, match="unsupported dtype"):
        binding.hsd_quantize_rows(f[0].double())
