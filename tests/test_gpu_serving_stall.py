"""The device-side timeout path of the FFN step in bf16, the one serving call whose kernels wait (bounded) for copies and matrix instructions: the host asks for the
fault injection; the call must return, report the wait that ran out, and leave the workspace usable."""
import pytest
import torch

from paper_2506_18145_b200 import binding as rb

from test_gpu_parity import _status_detail

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,Dm,F,E,K", [
    (1, 512, 1024, 4, 1),           # a part of the contracted index a block
    (5, 512, 2048, 4, 2),
    (64, 256, 2048, 1, 1),          # 64 columns, two passes of the down projection
    (64, 1024, 2048, 16, 2),        # several tiles a block
])
def test_stalled_ffn_step_is_reported(B, Dm, F, E, K):
    g = torch.Generator(device="cuda")
    g.manual_seed(B)
    normal = lambda shape, std: (torch.randn(shape, generator=g, device="cuda") * std).bfloat16()
    x, W_gu, W_down = normal((B, Dm), 1.0), normal((E, 2 * F, Dm), Dm ** -0.5), normal((E, Dm, F), F ** -0.5)
    idx = torch.topk(torch.rand((B, E), generator=g, device="cuda"), K, dim=1).indices.to(torch.int32).contiguous()
    gates = torch.rand((B, K), generator=g, device="cuda")
    good, stalled = (rb.make_config(B, 1, Dm, 64, 16, 4, 16, E, K, "bf16", flags=f) for f in (0, rb.ROM_FLAG_TEST_STALL))
    size = rb.ffn_moe_step_workspace_size(good, F)
    assert rb.ffn_moe_step_workspace_size(stalled, F) == size
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def call(cfg):
        out = torch.empty((B, Dm), dtype=torch.bfloat16, device="cuda")
        rb.rom_ffn_moe_step(cfg, F, W_gu, W_down, x, idx, gates, out, ws)
        torch.cuda.synchronize()
        return out

    ref = call(good)
    assert rb.rom_get_status(ws) == 0
    call(stalled)
    assert _status_detail(ws)[1] in (4, 5, 6, 7)
    assert rb.rom_get_status(ws) == -6
    assert torch.equal(call(good), ref) and rb.rom_get_status(ws) == 0
