"""Calls on caches held whole refuse every tensor of another device than the current one, which their kernels would run on (no GPU needed)."""
import pytest
import torch

from paper_2406_02542_amd import api


class Here(torch.Tensor):
    """A tensor that says it is one of device 1's."""
    __torch_function__ = torch._C._disabled_torch_function_impl
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 1


class There(Here):
    def get_device(self):
        return 0


class Launched(Exception):
    pass


class Library:
    def __getattr__(self, name):
        def call(*args):
            raise Launched
        return call


B, N, HQ, H, S = 2, 3, 4, 2, 32


def _tensors():
    i, f = torch.int32, torch.float32
    make = lambda shape, dt=f: torch.zeros(shape, dtype=dt).as_subclass(Here)
    return dict(cache_k=make((B, H, S, 128)), cache_v=make((B, H, S, 128)), rows=make((B, N), i), positions=make((B, N), i), frequencies=make((64,), torch.float64),
                k=make((B, N, H, 128)), v=make((B, N, H, 128)), q=make((B, N, HQ, 128)), q_out=make((B, N, HQ, 128)), out=make((B, N, HQ, 128)),
                k_out=make((B, H, N, 128)), v_out=make((B, H, N, 128)), seq_lens=make((B, N), i), workspace=make((1 << 20,), torch.uint8))


def _append(lay, t):
    c = api.Cache(lay, t["cache_k"], t["cache_v"])
    api.loki_append(lay, c, t["rows"], t["k"], t["v"], positions=t["positions"], frequencies=t["frequencies"], q=t["q"], q_out=t["q_out"])


def _read(lay, t):
    api.loki_read_rows(lay, api.Cache(lay, t["cache_k"], t["cache_v"]), t["rows"], t["k_out"], t["v_out"])


def _attend(lay, t):
    c = api.Cache(lay, t["cache_k"], t["cache_v"])
    api.dense_decode_cache(lay, c, t["q"], S, t["workspace"], t["out"], seq_lens=t["seq_lens"], queries_per_seq=N)


CALLS = [(_append, ("rows", "k", "v", "positions", "frequencies", "q", "q_out")), (_read, ("rows", "k_out", "v_out")), (_attend, ("q", "workspace", "out", "seq_lens"))]


@pytest.fixture
def second_device(monkeypatch):
    monkeypatch.setattr(api, "_current_device", lambda: 1)
    monkeypatch.setattr(api, "_current_raw_stream", lambda device: 0)
    monkeypatch.setattr(api, "lib", Library)
    return api.make_layout(B, HQ, H, 128, 128, S, torch.float32)


@pytest.mark.parametrize("call", [c for c, _ in CALLS])
def test_tensors_of_the_current_device_are_taken(second_device, call):
    with pytest.raises(Launched):
        call(second_device, _tensors())


@pytest.mark.parametrize("call,name", [(c, n) for c, names in CALLS for n in names])
def test_a_tensor_of_another_device_is_refused(second_device, call, name):
    t = _tensors()
    t[name] = t[name].as_subclass(There)
    with pytest.raises(ValueError, match=name + " must live on the current device"):
        call(second_device, t)


@pytest.mark.parametrize("call", [c for c, _ in CALLS])
def test_a_cache_of_another_device_is_refused(second_device, call):
    t = _tensors()
    for name in ("cache_k", "cache_v"):
        t[name] = t[name].as_subclass(There)
    with pytest.raises(ValueError, match="cache must live on the current device"):
        call(second_device, t)


def test_a_cache_of_two_devices_is_refused(second_device):
    t = _tensors()
    with pytest.raises(ValueError, match="same device"):
        api.Cache(second_device, t["cache_k"], t["cache_v"].as_subclass(There))
