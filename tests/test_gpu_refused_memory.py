"""Allocations that the device refuses: the call says so, and what comes after it on the same thread works as if it had not been."""
import pytest

from ._harness import log

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
LEFT = 2 << 30                # bytes that are left free while the calls ask for more


def test_a_refused_allocation_is_reported_once():
    import paper_2511_21702_amd as csv
    small = torch.randn(300, 64, device="cuda").to(torch.bfloat16)
    want = csv.csv_mx4_quantize(small)
    # inputs are whole, so that a call that does get its memory is an ordinary one
    codes, scales = torch.zeros(1 << 20, 4096, dtype=torch.uint8, device="cuda"), torch.zeros(1 << 20, 256, dtype=torch.uint8, device="cuda")
    W, b = torch.empty(1 << 18, 8192, dtype=torch.bfloat16, device="cuda").normal_(), torch.zeros(1 << 18, device="cuda")
    thin = torch.empty(4000003, 8, dtype=torch.bfloat16, device="cuda").normal_()
    idx = csv.csv_build_index(thin, None, 8)
    calls = {"head": lambda: csv.csv_mx4_head(codes, scales, None, 8192),     # 4.5 GB of bands
             "index": lambda: csv.csv_build_index(W, b, 8),                   # a copy of 4.3 GB
             "workspace": lambda: csv.CsvWorkspace(idx, 256, 8)}              # 4.1 GB of logits
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    hold = torch.empty(max(torch.cuda.mem_get_info()[0] - LEFT, 0), dtype=torch.uint8, device="cuda")
    try:
        for what, ask in calls.items():
            log(f"refused memory: {what}")
            with pytest.raises(csv.CsvError) as e:
                ask()
            assert e.value.code == -2 and "memory" in str(e.value)
            got = csv.csv_mx4_quantize(small)              # with the error still fresh: it is not this launch's
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    finally:
        del hold
        torch.cuda.empty_cache()
    for what, ask in calls.items():                        # and with memory to be had
        log(f"granted memory: {what}")
        ask().free()
    idx.free()
    del codes, scales, W, b, thin
    torch.cuda.empty_cache()
