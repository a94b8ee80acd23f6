"""A bounded wait that runs out in an operator on the caller's stream: reported once by the operators' own
status, apart from the sampler's."""

import pytest
import torch

from paper_2608_09231_gb300 import bag, configs, lowbit, synth

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_expired_wait_of_an_operator(lib):
    cfg = configs.get_config("tiny")
    ctx = bag.create(cfg, T=4, B=2)
    ctx.operators_status()
    ctx.check_operator_timeout()                    # enqueued: nothing is reported yet
    with pytest.raises(bag.BagError) as e:
        ctx.operators_status()
    assert e.value.status == 5 and "caller's stream" in str(e.value)
    ctx.operators_status()                          # reported, cleared
    # the sampler has no part in it
    ctx.check_operator_timeout()
    inp = synth.make_inputs(cfg)
    x, txt, pooled = (torch.from_numpy(inp[n].copy()).to(DEV) for n in ("x", "txt", "pooled"))
    txt = txt.to(torch.bfloat16) if cfg["dtype"] == "bf16" else txt
    mask, _, nfe = ctx.run(x, txt, pooled)
    assert nfe == 2 and int(mask.sum()) == 2 and bool(torch.isfinite(x).all())
    # nor does the sampler's own error reach, or clear, the operators'
    assert ctx.check_wait_timeout() == 5
    ctx.reset()
    with pytest.raises(bag.BagError) as e:
        ctx.operators_status()
    assert e.value.status == 5
    assert ctx.check_wait_timeout() == 5
    ctx.operators_status()
    ctx.close()


def test_a_sample_of_the_block_reports_it(lib):
    ctx = bag.create("tiny", T=2, B=1)
    block = lowbit.LowBitBlock(ctx, lowbit.random_weights(256, 512), 300, keep=2)
    h0 = torch.randn(300, 256, device=DEV)
    outs = [torch.empty_like(h0) for _ in range(2)]
    mod = [0.5 * torch.randn(256, device=DEV) for _ in range(6)]
    block.run([h0, h0], outs, [mod] * 2, [1, 0])
    ctx.check_operator_timeout()
    with pytest.raises(bag.BagError) as e:
        block.run([h0, h0], outs, [mod] * 2, [1, 0])
    assert e.value.status == 5
    block.run([h0, h0], outs, [mod] * 2, [1, 0])
    ctx.close()


def test_status_while_the_stream_is_captured(lib):
    """Refused, and the capture goes on; a whole sample may be captured."""
    ctx = bag.create("tiny", T=2, B=1)
    block = lowbit.LowBitBlock(ctx, lowbit.random_weights(256, 512), 300, keep=2)
    h0 = torch.randn(300, 256, device=DEV)
    want, outs = ([torch.empty_like(h0) for _ in range(2)] for _ in range(2))
    mod = [0.5 * torch.randn(256, device=DEV) for _ in range(6)]
    block.run([h0, h0], want, [mod] * 2, [1, 0])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx.set_stream(s.cuda_stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            block.run([h0, h0], outs, [mod] * 2, [1, 0])
            with pytest.raises(bag.BagError) as e:
                ctx.operators_status()
            assert e.value.status == 6
        graph.replay()
        ctx.operators_status()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    ctx.close()
