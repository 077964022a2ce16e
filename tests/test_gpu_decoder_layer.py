"""The example: a decoder layer with compressed weights gives the same for a prompt as for its tokens one by one, with and without a
window, and for sequences that share the prompt as their prefix."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder_layer.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("decoder_layer_example", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def close(a, b):
    # both ways round to bf16 some ten times between input and output (norms, heads, weights of the attention, activations, products of
    # the prompt), each 2^-9 of a value at most on average: 10 roundings that add like independent ones, and three times that
    return float((a - b).norm() / b.norm()) <= 3 * 10 ** 0.5 * 2.0 ** -9


@pytest.mark.parametrize("heads,kv_heads,window,sinks", [(4, 4, 0, 0), (8, 2, 0, 0), (8, 1, 50, 4)])
def test_tokens_one_by_one_give_what_the_prompt_gives(example, heads, kv_heads, window, sinks):
    n, hidden = 150, 512
    print(f"case layer heads={heads}/{kv_heads} window={window}", flush=True)
    layer = example.DecoderLayer(hidden, heads, kv_heads, 1024, 8, n, window, sinks, seed=3)
    x = torch.randn(n, hidden, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    table = [[5, 0, 3]]
    whole = layer.prompt(x, example.batch_of([n], [n], table))
    k, v = layer.k_pool.clone(), layer.v_pool.clone()
    layer.k_pool.zero_()
    layer.v_pool.zero_()
    layer.prompt(x[:100], example.batch_of([100], [100], table))
    tokens = torch.cat([layer.token(x[t:t + 1], example.batch_of([t + 1], [1], table)) for t in range(100, n)])
    torch.cuda.synchronize()
    assert close(tokens, whole[100:])
    assert close(layer.k_pool.float(), k.float()) and close(layer.v_pool.float(), v.float())


def test_sequences_behind_a_common_prefix(example):
    n, hidden, tail = 100, 512, 30
    print("case layer prefix", flush=True)
    layer = example.DecoderLayer(hidden, 8, 2, 1024, 16, 200, seed=4)
    x = torch.randn(n + 3 * tail, hidden, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda")
    layer.prompt(x[:n], example.batch_of([n], [n], [[1, 2]]))
    # three continuations of it, whose own tokens lie in pages of their own
    own = [[7], [4], [9]]
    lens = [n + tail] * 3
    together = layer.prompt(x[n:], example.batch_of(lens, [tail] * 3, own, n, [1, 2]))
    for b in range(3):
        alone = torch.cat([x[:n], x[n + b * tail:n + (b + 1) * tail]])
        want = layer.prompt(alone, example.batch_of([n + tail], [n + tail], [[10, 11, 12]]))[n:]
        assert close(together[b * tail:(b + 1) * tail], want)
