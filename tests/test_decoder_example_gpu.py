"""The example decoder runs the norm, the cache and the attention together with the linear layers:
a prompt in one call, in two parts and token by token gives the same hidden states."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decoder_layers.py")
    spec = importlib.util.spec_from_file_location("decoder_layers", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 2)])
def test_prompt_in_parts_and_token_by_token(example, window, sinks):
    n, cut, d = 61, 40, 512
    # 8-bit activations everywhere: a code that a rounding moves shifts a value by under 1 %
    kw = dict(layers=2, d=d, heads=8, kv_heads=2, f=768, mask_a8=(0, 1), pages=32, window=window, sinks=sinks)
    x = torch.randn((n, d), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").half()
    whole = example.Decoder(**kw).step(x, {0: n})
    two = example.Decoder(**kw)
    parts = torch.cat([two.step(x[:cut], {0: cut}), two.step(x[cut:], {0: n - cut})])
    one = example.Decoder(**kw)
    single = torch.cat([one.step(x[i:i + 1], {0: 1}) for i in range(n)])
    # Pages filled in parts carry the same scales but may hold codes one off (their rows were
    # rescaled as the scale grew): half a step of 1/127 of a page's largest value each time, at
    # most four or five times for random rows, averaged over the keys by the softmax.
    for got in (parts, single):
        err = (got.float() - whole.float()).norm(dim=1) / whole.float().norm(dim=1)
        assert err.max() < 0.05 and err.mean() < 0.02
    # other sequences in the batch change nothing
    both = example.Decoder(**kw).step(torch.cat([x[:17], x]), {7: 17, 0: n})[17:]
    err = (both.float() - whole.float()).norm(dim=1) / whole.float().norm(dim=1)
    assert err.max() < 0.05


def test_example_runs(example, capsys):
    example.main()
    assert "decode: 32 steps" in capsys.readouterr().out
