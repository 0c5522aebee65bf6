"""Norms of other widths called from two host threads at a time: one thread's launches take nothing from the other's. The widths of a pair
share a kernel and differ in the shared memory that they ask for."""
import threading

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_22755_b200 import binding

    return binding


@pytest.mark.parametrize("dtype,dims,backward", [("bf16", (5511, 8191), True), ("f32", (5001, 8001), True), ("bf16", (7001, 8191), False),
                                                 ("f32", (9001, 16383), False), ("bf16", (520, 1024), True)])
def test_two_threads(B, dtype, dims, backward):
    import torch

    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    calls = []
    for dim in dims:
        g = torch.Generator("cuda").manual_seed(dim)
        x, dy = (torch.randn(3, dim, generator=g, device="cuda").to(dt) for _ in range(2))
        w, mean, rstd = torch.randn(dim, generator=g, device="cuda"), torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
        y, dw = torch.empty_like(x), torch.empty(dim, device="cuda")
        ws = torch.empty(B.nsp_norm_bwd_ws_bytes(3, dim), dtype=torch.uint8, device="cuda")
        stream = torch.cuda.Stream()
        B.nsp_norm_fwd(x, w, None, y, mean, rstd)

        # the library's own entry, so that the threads spend their time there and not on Python's lock
        rows = [B._ROWS.pack(t.data_ptr(), dim, 0) for t in (x, dy, y)]
        code, ptr = B.NSP_F32 if dt == torch.float32 else B.NSP_BF16, lambda t: t.data_ptr()
        if backward:
            args = (rows[0], rows[1], ptr(w), ptr(mean), ptr(rstd), rows[2], ptr(dw), None, 3, 1, dim, code, B.NSP_F32, B.NSP_NORM_LAYER, ptr(ws),
                    ws.numel(), stream.cuda_stream)
        else:
            args = (rows[0], ptr(w), None, rows[2], ptr(mean), ptr(rstd), 3, 1, dim, code, B.NSP_F32, B.NSP_NORM_LAYER, 1e-5, stream.cuda_stream)
        entry = B.lib().nsp_norm_bwd if backward else B.lib().nsp_norm_fwd
        torch.cuda.synchronize()
        assert entry(*args) == B.NSP_OK
        torch.cuda.synchronize()
        calls.append((entry, args, (y, dw), (y.clone(), dw.clone()), (x, dy, w, mean, rstd, ws, stream)))
    wrong = []

    def go(entry, args):
        wrong.extend(rc for rc in (entry(*args) for _ in range(10000)) if rc != B.NSP_OK)

    threads = [threading.Thread(target=go, args=c[:2]) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong, f"{len(wrong)} of 20,000 calls failed"
    for _, _, got, want, _ in calls:
        assert torch.equal(got[0], want[0]) and (not backward or torch.equal(got[1], want[1]))
