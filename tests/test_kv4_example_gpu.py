"""The example decoder on the 4-bit cache with rotary positions from the library: a prompt in one call, in two parts and token
by token gives the same hidden states; its rotary positions are those of a plain form."""
import pytest

from test_decoder_example_gpu import example  # noqa: F401  (the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks,rotary", [(0, 0, {}), (24, 2, dict(scaling="wavelength", factor=4.0, trained_len=32.0))])
def test_prompt_in_parts_and_token_by_token(example, window, sinks, rotary):  # noqa: F811
    n, cut, d = 61, 40, 512
    kw = dict(layers=2, d=d, heads=8, kv_heads=2, f=768, mask_a8=(0, 1), pages=32, window=window, sinks=sinks, kv_bits=4,
              rotary=rotary)
    x = torch.randn((n, d), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").half()
    whole = example.Decoder(**kw).step(x, {0: n})
    two, one = example.Decoder(**kw), example.Decoder(**kw)
    parts = torch.cat([two.step(x[:cut], {0: cut}), two.step(x[cut:], {0: n - cut})])
    single = torch.cat([one.step(x[i:i + 1], {0: 1}) for i in range(n)])
    # The first layer's cache is the same bit for bit (below).  Its attention differs by binary16 roundings, of which 8-bit
    # codes behind them make e = 0.005 of a row: delta = 2^-11 v moves a code by its step (1 / 127 of 3 sigma, 0.024 sigma)
    # with probability delta / step = 0.02, 0.0034 in the mean square, twice a layer.  The second layer's 4-bit codes
    # have steps s = max / 7 = 0.39 sigma (64 values: a maximum of 2.7 sigma): a value moved by delta takes another code with
    # probability |delta| / s, so its mean square change is E|delta| s = 0.8 e 0.39 sigma^2 = 0.0016 sigma^2, 0.039 of a row of K
    # and of V.  Logits (of unit variance) move by 0.039, and so do their weights: with V's own, 0.056 of that
    # attention's output, which is at most half of the hidden state: 0.028, and e: 0.033 on average.
    for got in (parts, single):
        err = (got.float() - whole.float()).norm(dim=1) / whole.float().norm(dim=1)
        assert err.max() < 0.05 and err.mean() < 0.035
    both = example.Decoder(**kw).step(torch.cat([x[:17], x]), {7: 17, 0: n})[17:]
    err = (both.float() - whole.float()).norm(dim=1) / whole.float().norm(dim=1)
    assert err.max() < 0.05


def test_first_layers_caches_agree(example):  # noqa: F811
    kw = dict(layers=1, d=512, heads=8, kv_heads=2, f=768, mask_a8=(0,), pages=32, kv_bits=4)
    x = torch.randn((50, 512), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").half()
    a, b = example.Decoder(**kw), example.Decoder(**kw)
    a.step(x, {0: 50})
    for i in range(0, 50, 7):
        b.step(x[i:i + 7], {0: min(7, 50 - i)})
    ca, cb = a.layers[0]["cache"], b.layers[0]["cache"]
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert torch.equal(getattr(ca, name)[a.tables[0]], getattr(cb, name)[b.tables[0]])


def test_example_runs_on_the_4_bit_cache(example, capsys):  # noqa: F811
    example.main(kv_bits=4)
    assert "decode: 32 steps" in capsys.readouterr().out
