"""Bounded waits of the operators that run out: they are reported, and what was not computed is not taken for a result.  The kernels are
built here with a limit of a millisecond."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2510_19705_b200 import binding, build

pytestmark = pytest.mark.gpu
vp, i32, c_float, size_t = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
HERE = os.path.dirname(os.path.abspath(__file__))


def native(tmp_path_factory, name, *more):
    if not os.path.exists(build.NVCC):
        pytest.skip("no nvcc")
    out = str(tmp_path_factory.mktemp("native") / (name + ".so"))
    sources = [os.path.join(HERE, "native", name + ".cu")] + [os.path.join(build.CSRC, m) for m in more]
    subprocess.run([build.NVCC] + build.FLAGS + ["-DHSD_WAIT_LIMIT_NS=1000000ull", "-shared", "-Xlinker", "-Bsymbolic", "-o", out] + sources +
                   ["-L" + build.HERE, "-l:libhsd.so", "-Xlinker", "-rpath," + build.HERE], check=True)
    return ctypes.CDLL(out)


@pytest.fixture(scope="module")
def prefix(lib, tmp_path_factory):
    lib.library()
    so = native(tmp_path_factory, "prefix_waits", "attn_prefix.cu")
    so.hsd_prefix_attention.argtypes = binding.library().hsd_prefix_attention.argtypes
    return so


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# a warp or eight a row and head in the join; one query tile, several
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("rows,nq", [(20, 4), (20, 32), (300, 8)])
def test_prefix_attention_whose_waits_run_out(lib, prefix, hd, rows, nq):
    P, stream = 200, torch.cuda.current_stream().cuda_stream
    q = torch.randn(rows, nq, hd, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn(2, 40, 16, hd, device="cuda").to(torch.bfloat16) for _ in range(2))
    table, lens = ints([[-1] * 12 + [20]] * rows), ints([P + 1] * (rows - 1) + [0])
    pages, length = ints(list(range(13)) + [-1] * 400000), ints([P])
    ws = torch.full((lib.hsd_prefix_attention_workspace_bytes(rows, nq, 2, hd),), 0x7F, dtype=torch.uint8, device="cuda")       # places that are none
    out = torch.zeros_like(q)
    pool = binding._KvPool(k=k.data_ptr(), v=v.data_ptr(), dtype=1, n_pages=40, page_size=16, head_stride=k.stride(0), page_stride=k.stride(1), token_stride=k.stride(2))
    assert prefix.hsd_prefix_attention(q.data_ptr(), rows, nq, 2, hd, ctypes.byref(pool), table.data_ptr(), 13, lens.data_ptr(), None, rows, pages.data_ptr(), len(pages),
                                       length.data_ptr(), 0.1, ws.data_ptr(), ws.numel(), 1, out.data_ptr(), stream) == 0
    status = binding.library().hsd_gemm_status(ws.data_ptr(), stream)
    assert status == -5                                                     # HSD_E_DEVICE_TIMEOUT
    assert bool(out.isnan().all())
    # the same workspace serves the next call
    args = (q, k, v, table, lens, pages, length)
    assert torch.equal(lib.hsd_prefix_attention(*args, workspace=ws), lib.hsd_prefix_attention(*args))
    assert binding.library().hsd_gemm_status(ws.data_ptr(), stream) == 0


@pytest.fixture(scope="module")
def w8(lib, tmp_path_factory):
    lib.library()
    so = native(tmp_path_factory, "w8_waits")
    so.w8_without_data.argtypes = [vp, vp, i32, i32, vp, vp, i32, vp, i32, vp, vp]
    return so


# K by clusters of eight, four and two, by CTAs of their own with one tile and with several; CTA pairs with one tile and with several
@pytest.mark.parametrize("R,N,K", [(3, 1000, 2048), (16, 2000, 2048), (200, 5000, 512), (1, 18000, 256), (250, 40000, 128), (300, 500, 256), (1000, 12000, 128)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_products_whose_waits_run_out(lib, w8, R, N, K, dtype):
    a, w = (torch.ones(n, K, dtype=torch.int8, device="cuda") for n in (R, N))
    rows, cols, status = torch.ones(R, device="cuda"), torch.ones(N, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    out, stream = torch.zeros(R, N, dtype=dtype, device="cuda"), torch.cuda.current_stream().cuda_stream
    assert w8.w8_without_data(a.data_ptr(), rows.data_ptr(), R, K, w.data_ptr(), cols.data_ptr(), N, out.data_ptr(), 0 if dtype == torch.float32 else 1, status.data_ptr(), stream) == 0
    torch.cuda.synchronize()
    assert int(status) == 1 and bool(out.isnan().all())


def test_calls_that_are_asked_to_report_waits_that_gave_up(lib):
    """check=True on whole calls, and with a status call that answers with the error."""
    g = torch.randn(40, 8, 64, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn(2, 4, 16, 64, device="cuda").to(torch.bfloat16) for _ in range(2))
    prefix_args = (g, k, v, ints([[2, 3]] * 40), ints([20] * 40), ints([0, 1]), ints([17]))
    codes, scales = lib.hsd_quantize_rows(torch.randn(100, 512, device="cuda"))
    calls = (lambda **c: lib.hsd_prefix_attention(*prefix_args, **c), lambda **c: lib.hsd_gemm_w8(g.view(40, -1), codes, scales, **c))
    for call in calls:
        assert torch.equal(call(check=True), call())
    asked = []
    fake = ctypes.CFUNCTYPE(i32, vp, vp)(lambda workspace, stream: asked.append(workspace) or -5)
    library = binding.library()
    real, binding._host = library.hsd_gemm_status, None
    try:
        library.hsd_gemm_status = fake
        binding._host_calls()
        for i, call in enumerate(calls):
            with pytest.raises(binding.HsdError, match="timed out"):
                call(check=True)
            assert len(asked) == i + 1 and asked[i] % 256 == 0
            call()
            assert len(asked) == i + 1                                      # not asked, not waited for
    finally:
        library.hsd_gemm_status, binding._host = real, None
        binding._host_calls()
    for call in calls:
        call(check=True)
