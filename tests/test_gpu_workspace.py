"""GPU: a caller's workspace is refused where a kernel could not write to it, before anything is launched."""
import pytest

torch = pytest.importorskip("torch")
import paper_2504_13989_amd as rq  # noqa: E402
from paper_2504_13989_amd import binding  # noqa: E402

pytestmark = pytest.mark.gpu

WORDS = 1 << 16


def calls():
    g = torch.Generator(device="cuda").manual_seed(0)
    x, h = torch.randn(64, 1024, generator=g, device="cuda"), rq.hadamard_build(1024)
    yield "quant_error", lambda ws: binding.quant_error(h, x, 4, [0.9, 1.0], workspace=ws)
    yield "gbs_search", lambda ws: torch.tensor(rq.gbs_search(h, x, 4, 0.01, workspace=ws)[:2])
    cache, hk = rq.kv4_cache(128, 1, 64, 64), rq.hadamard_build(64)
    k, slots = torch.randn(8192, 1, 64, generator=g, device="cuda"), torch.arange(8192, device="cuda")
    rq.kv4_append(hk, cache, k, k, slots)
    q = torch.randn(1, 8, 64, generator=g, device="cuda").bfloat16()
    table, lens = torch.arange(128, dtype=torch.int32, device="cuda")[None], torch.tensor([8192], dtype=torch.int32, device="cuda")
    yield "kv4_attention", lambda ws: rq.kv4_attention(hk, cache, q, table, lens, workspace=ws)


def test_workspaces_that_cannot_be_written_to_are_refused():
    bad = [torch.empty(WORDS * 64, dtype=torch.float64), torch.empty(1, dtype=torch.float64, device="cuda").expand(WORDS * 64),
           torch.empty(2 * WORDS, dtype=torch.float64, device="cuda")[::2], torch.empty(WORDS, dtype=torch.float64, device="meta")]
    for name, call in calls():
        for ws in bad:
            with pytest.raises(ValueError):
                call(ws)
        with pytest.raises(TypeError):
            call(WORDS)


def test_workspaces_that_hold_the_call_are_taken():
    for name, call in calls():
        want = call(None)
        big = torch.empty(WORDS * 64, dtype=torch.float64, device="cuda")
        for ws in (big, big.view(WORDS, 64).t()):
            assert torch.equal(torch.as_tensor(call(ws)), torch.as_tensor(want)), name
