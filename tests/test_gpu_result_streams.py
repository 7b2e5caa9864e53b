"""New results of the stage and of the model's ends on a named stream: memory of that stream's pool, and the same bits."""
import pytest
import torch

from harness import gpu_stage, to_dev
from paper_2505_21070_amd import synth
from test_gpu_ends import make_ends
from test_gpu_paged_streams import pool_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["tiny", "small_bf16"])
def test_results_of_a_named_stream(name):
    cfg, w, text, blocks = synth.make_case(name, seed=3, strong_gate=True)
    nf, nc = cfg["block_frames"], cfg["cache_frames"]
    g = gpu_stage(cfg, w, text)
    ends, _ = make_ends(cfg, w, 16, nf)
    lat = synth.make_latent(cfg, nf, 16, torch.Generator().manual_seed(2)).cuda()
    x = to_dev(blocks[1], cfg)
    g.forward(to_dev(blocks[0], cfg), nf, nf, 625.0)
    g.cache_update(0, nc)

    def results(stream):
        y = g.forward(x, nf, 0, 500.0, stream=stream)
        return y, g.peek("k", stream=stream), ends.embed(lat, stream=stream), ends.head(y, 437.0, nf, stream=stream)
    want = results(None)
    torch.cuda.synchronize()
    here, side = torch.cuda.current_stream().cuda_stream, torch.cuda.Stream()
    for stream, pool in ((side, side.cuda_stream), (None, here), (side, side.cuda_stream)):
        got = results(stream)
        torch.cuda.synchronize()
        assert [pool_of(t.data_ptr()) for t in got] == [pool] * 4
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del got


def test_handles_made_on_a_named_stream():
    """Their workspaces, which init writes, too."""
    from paper_2505_21070_amd import binding as B
    cfg, w, text, blocks = synth.make_case("tiny", seed=3, strong_gate=True)
    nf = cfg["block_frames"]
    side = torch.cuda.Stream()
    weights, words, x = B.weights_to_device(w, cfg["dtype"]), text.to("cuda").contiguous(), to_dev(blocks[0], cfg)
    side.wait_stream(torch.cuda.current_stream())
    a = B.Stage(B.make_config(cfg, max_abs_frames=16), weights, words)
    b = B.Stage(B.make_config(cfg, max_abs_frames=16), weights, words, stream=side)
    ends, _ = make_ends(cfg, w, 4, nf)
    assert pool_of(ends.workspace.data_ptr()) == pool_of(a.workspace.data_ptr()) == torch.cuda.current_stream().cuda_stream
    assert pool_of(B.Ends(cfg, ends._keep, 4, nf, stream=side).workspace.data_ptr()) == pool_of(b.workspace.data_ptr()) == side.cuda_stream
    want = a.forward(x, nf, nf, 625.0)
    got = b.forward(x, nf, nf, 625.0, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
