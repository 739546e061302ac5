"""The operators' bindings refuse tensors that do not lie on the context's device, before anything is called."""
import ctypes
import types

import pytest
import torch

import paper_2609_03949_amd as vkv

BF, I32 = torch.bfloat16, torch.int32


class Refused:
    """In libvkv's place: every call has been one too many."""

    def __getattr__(self, name):
        def call(*args):
            raise AssertionError(f"{name} was called")
        return call


@pytest.fixture()
def ctx():
    return types.SimpleNamespace(device=0, lib=Refused(), handle=None, check=lambda rc: None)


def tensors(dev):
    z = lambda *s, t=BF: torch.zeros(*s, dtype=t, device=dev)
    return types.SimpleNamespace(
        q=z(5, 4, 128), k=z(5, 2, 128), v=z(5, 2, 128), cu=torch.tensor([0, 5], dtype=I32, device=dev), out=z(5, 4, 128),
        lse=z(5, 4, t=torch.float32), cache=z(3, 16, 576), table=z(1, 2, t=I32), kv=z(1, t=I32), ql=z(5, 4, 512), qr=z(5, 4, 64),
        out2=z(5, 4, 512), ws=z(1 << 24, t=torch.uint8), weight=z(1, 32, t=torch.float32), kept=z(1, 4, t=I32), count=z(1, t=I32),
        origin=z(1, 4, t=I32), moved=z(1, 4, t=torch.float32))


def calls(ctx, t, stream=None, **other):
    """Each operator's call; `other` replaces tensors of the calls themselves."""
    pr = vkv.Prompt(t.q, t.k, t.v, t.cu, 5)
    pages, chunk = vkv.Pages(t.cache, t.table, t.kv, 32), vkv.Chunk(t.ql, t.qr, t.cu, 5)
    t = types.SimpleNamespace(**dict(vars(t), **other))
    return dict(
        prompt=lambda: vkv.prompt_attend(ctx, pr, 0.1, t.out, t.lse, stream),
        chunk=lambda: vkv.chunk_attend(ctx, pages, chunk, t.ws, 0.1, t.out2, t.lse, stream),
        weights=lambda: vkv.weight_accumulate(ctx, pages, chunk, t.lse, t.ws, 0.1, 0.5, t.weight, t.weight, stream),
        select=lambda: vkv.weight_select(ctx, t.weight, t.kv, 32, 0, 0, t.kept, t.count, stream),
        evict=lambda: vkv.cache_evict(ctx, pages, t.kept, t.count, t.origin, t.weight, t.moved, stream))


NAMES = ("prompt", "chunk", "weights", "select", "evict")


@pytest.mark.parametrize("name", NAMES)
def test_host_tensors_are_refused(ctx, name):
    with pytest.raises(ValueError, match="device"):
        calls(ctx, tensors("cpu"))[name]()


def test_descriptions_of_tensors_on_several_devices(ctx):
    t = tensors("cpu")
    fake = types.SimpleNamespace
    for make in (lambda x: vkv.Prompt(x.q, x.k, x.v, x.cu, 5), lambda x: vkv.Pages(x.cache, x.table, x.kv, 32),
                 lambda x: vkv.Chunk(x.ql, x.qr, x.cu, 5)):
        assert make(t).device == -1
    assert vkv._one_device(t.q, None, t.cu) == -1
    with pytest.raises(ValueError, match="different devices"):
        vkv._one_device(fake(get_device=lambda: 0, device="cuda:0"), fake(get_device=lambda: 1, device="cuda:1"))
    a, b = vkv.Pages(t.cache, t.table, t.kv, 32), vkv.Chunk(t.ql, t.qr, t.cu, 5)
    b.device = 0
    with pytest.raises(ValueError, match="different devices"):
        vkv.chunk_workspace_size(a, b)


def test_streams_of_another_device(ctx):
    other = types.SimpleNamespace(device=torch.device("cuda:1"), cuda_stream=0)
    with pytest.raises(ValueError, match="stream"):
        vkv._call_stream(ctx, other, 0)
    assert vkv._call_stream(ctx, types.SimpleNamespace(device=torch.device("cuda:0"), cuda_stream=77), 0) == 77
    with pytest.raises(ValueError, match="cuda:1"):
        vkv._call_stream(ctx, other, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_each_tensor_of_a_call(ctx, name):
    """On the device, with one of the call's tensors in host memory."""
    t, h = tensors("cuda"), tensors("cpu")
    own = dict(prompt=("out", "lse"), chunk=("ws", "out2", "lse"), weights=("lse", "ws", "weight"),
               select=("weight", "kv", "kept", "count"), evict=("kept", "count", "origin", "weight", "moved"))[name]
    for one in own:
        with pytest.raises(ValueError, match="device"):
            calls(ctx, t, **{one: getattr(h, one)})[name]()
    real = vkv.Context(0)
    calls(real, t)[name]()
    calls(real, t, stream=torch.cuda.current_stream())[name]()
    torch.cuda.synchronize()
