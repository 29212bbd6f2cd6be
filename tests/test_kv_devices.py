"""Tensors of a cache, a batch or a call that are on several devices, or not on the current one, are refused before anything is
launched (stand-ins for tensors: no GPU needed)."""
import pytest

torch = pytest.importorskip("torch")


class Tensor:
    """What the binding looks at of a CUDA tensor."""
    is_cuda = True

    def __init__(self, dtype, *shape, device=0):
        self.dtype, self.shape, self.device = dtype, shape, device

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def stride(self):
        st = [1]
        for n in self.shape[:0:-1]:
            st.insert(0, st[0] * n)
        return tuple(st)

    def get_device(self):
        return self.device

    def data_ptr(self):
        return 64


@pytest.fixture
def dp(monkeypatch):
    from paper_2606_12487_gb300 import dptq
    dptq.load()
    dptq._HALF = torch.float16
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    return dptq


def _batch(dp, devices=(0, 0, 0), tokens=0):
    i = torch.int32
    return dp.Kv8Batch(Tensor(i, 3, device=devices[0]), Tensor(i, 2, device=devices[1]), Tensor(i, 2, 5, device=devices[2]),
                       tokens=tokens, max_tokens=tokens, max_len=80)


def _cache(dp, bits, devices=(0, 0, 0, 0)):
    if bits == 8:
        codes, scales = (torch.int8, 10, 2, 16, 64), (torch.float32, 10, 2)
        cls = dp.Kv8Cache
    else:
        codes, scales = (torch.uint8, 10, 2, 16, 32), (torch.bfloat16, 10, 2, 16)
        cls = dp.Kv4Cache
    return cls(*(Tensor(*shape, device=d) for shape, d in zip((codes, codes, scales, scales), devices)))


@pytest.mark.parametrize("at", range(3))
def test_a_batch_on_two_devices(dp, at):
    with pytest.raises(ValueError, match="one device"):
        _batch(dp, [int(i == at) for i in range(3)])
    assert _batch(dp, (1, 1, 1)).device == 1


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("at", range(4))
def test_a_cache_on_two_devices(dp, bits, at):
    with pytest.raises(ValueError, match="one device"):
        _cache(dp, bits, [int(i == at) for i in range(4)])
    assert _cache(dp, bits, (1, 1, 1, 1)).device == 1


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("wrong", [None, "cache", "batch", "first", "second"])
def test_a_call_on_another_device_than_the_current_one(dp, bits, wrong):
    on = {w: int(w == wrong) for w in ("cache", "batch", "first", "second")}
    # (a batch without tokens: the call that is in order launches nothing)
    cache, batch = _cache(dp, bits, [on["cache"]] * 4), _batch(dp, [on["batch"]] * 3)
    rows = [Tensor(torch.float16, 0, 2, 64, device=on[w]) for w in ("first", "second")]
    append, attention = (dp.dptq_kv8_append, dp.dptq_kv8_attention) if bits == 8 else (dp.dptq_kv4_append, dp.dptq_kv4_attention)
    calls = [lambda: append(cache, batch, *rows), lambda: attention(cache, batch, *rows, 0.1)]
    if bits == 4:
        calls.append(lambda: dp.dptq_kv4_read(cache, batch, *rows))
    for call in calls:
        if wrong is None:
            call()
        else:
            with pytest.raises(ValueError, match="current device"):
                call()
