"""The memory that a Cache holds beside its tensors: what its calls so far need."""
import ctypes

import pytest
import torch

from tests import test_gpu_new_rows as rows_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_37617_gb300 as p
    return p


def needs(lib, cache, *names):
    n = ctypes.c_int64()
    sizes = []
    for name in names:
        assert getattr(lib._lib, name)(cache._ref, ctypes.byref(n)) == 0
        sizes.append(n.value)
    return max(sizes)


def test_prompts_workspace_is_made_with_the_first_prompt(lib):
    x = rows_of.Prompt((28, 4, 128), [2000, 10], [40, 3])  # (cut along the keys: parts in the workspace)
    want, want_lse = rows_of.prompt(lib, x)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    cache = lib.Cache(x.k, x.v)
    made = torch.cuda.memory_allocated() - before
    others = needs(lib, cache, "as2d_tree_attention_workspace", "as2d_cache_evict_workspace")
    assert others <= made < others + 2 ** 20
    lse = torch.empty_like(want_lse)
    calls = [dict(), dict(), dict(stream=torch.cuda.Stream().cuda_stream)]
    for i, kw in enumerate(calls):
        lse.zero_()
        torch.cuda.synchronize()
        out = cache.prompt_attention(x.q, x.kv_len, x.rows, scale=x.scale, lse=lse, **kw)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        held = torch.cuda.memory_allocated() - before - made - lse.numel() * 4
        of_prompts = needs(lib, cache, "as2d_prompt_attention_workspace")
        assert of_prompts <= held < of_prompts + 2 ** 20 + out.numel() * 2
        del out


def test_prompts_workspace_first_on_another_stream(lib):
    """The first prompt on a stream of the caller's, captured, or on a stream of torch's; later ones
    elsewhere."""
    x = rows_of.Prompt((28, 4, 128), [2000, 10], [40, 3])
    want, _ = rows_of.prompt(lib, x)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    call = lambda cache, **kw: cache.prompt_attention(x.q, x.kv_len, x.rows, scale=x.scale, **kw)  # noqa: E731
    handle, captured, other = (lib.Cache(x.k, x.v) for _ in range(3))
    torch.cuda.synchronize()
    outs = [call(handle, stream=side.cuda_stream)]
    side.synchronize()
    outs.append(call(handle))
    with torch.cuda.graph(graph):
        in_graph = call(captured)
    in_graph.zero_()
    graph.replay()
    torch.cuda.synchronize()
    outs += [in_graph.clone(), call(captured)]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        outs.append(call(other))
    side.synchronize()
    outs.append(call(other))
    graph.replay()
    torch.cuda.synchronize()
    outs.append(in_graph)
    for out in outs:
        assert torch.equal(out, want)
