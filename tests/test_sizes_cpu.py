"""Sizes and settings that a C int does not hold are refused by the wrappers, before anything is allocated or called."""
import pytest
import torch

import paper_2510_22641_gb300 as lib
from paper_2510_22641_gb300 import heads, lowbit

WRAP = 1 << 32


class Tensor:
    """What the wrappers look at of a CUDA tensor, with any shape."""
    is_cuda, device = True, torch.device("cuda", 0)

    def __init__(self, *shape, dtype=torch.float32, strides=None):
        self.shape, self.dtype = torch.Size(shape), dtype
        st = [1]
        for n in shape[:0:-1]:
            st.insert(0, st[0] * n)
        self._strides = strides or tuple(st)

    def stride(self, i=None):
        return self._strides if i is None else self._strides[i]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def get_device(self):
        return 0

    def data_ptr(self):
        return 1 << 40

    def is_contiguous(self):
        return True


@pytest.fixture(autouse=True)
def no_device(monkeypatch):
    """Nothing is called, and what is allocated has no memory."""
    def called(*a):
        raise AssertionError("the library was called")
    lib.build()
    for m in (lowbit, heads):
        monkeypatch.setattr(m, "_call", called)
    monkeypatch.setattr(torch, "empty", lambda size, dtype=None, device=None: Tensor(*([size] if isinstance(size, int) else size),
                                                                                      dtype=dtype))


def made(cls, **fields):
    """An object as its constructor leaves it, without the packing."""
    o = object.__new__(cls)
    o.__dict__.update(lib=lowbit.B.load(), device=Tensor.device, _index=0, _packed=1 << 41, **fields)
    return o


def refused(f):
    with pytest.raises(lib.SSDError) as e:
        f()
    assert e.value.status == 1


@pytest.mark.parametrize("rows,k", [(WRAP + 5, 16), (5, WRAP + 16), (1 << 31, 16)])
def test_rows_to_pack(rows, k):
    refused(lambda: lib.F4Rows(Tensor(rows, k)))
    refused(lambda: lib.F4Weight(Tensor(rows, k)))
    refused(lambda: lib.W4Weight(Tensor(rows, k)))


def test_group_of_a_weight():
    refused(lambda: lib.W4Weight(Tensor(64, 256), group=WRAP + 64))


@pytest.mark.parametrize("rows", [WRAP, WRAP + 1, WRAP + 5, 1 << 31])
def test_rows_of_a_product(rows):
    w = made(lib.F4Weight, n=64, k=32, shape=torch.Size((64, 32)))
    refused(lambda: w.matmul(Tensor(rows, 32)))
    w = made(lib.W4Weight, n=64, k=128, group=64, _work=0)
    refused(lambda: w.matmul(Tensor(rows, 128)))
    refused(lambda: w.matmul(Tensor(rows, 128, dtype=torch.bfloat16)))


@pytest.mark.parametrize("shape", [(WRAP + 5, 4, 64), (5, WRAP + 4, 64), (1 << 31, 1, 64)])
def test_rows_and_heads_to_turn(shape):
    r = lib.Rotary(64)
    pos = Tensor(shape[0], dtype=torch.int32)
    refused(lambda: r.rotate(Tensor(*shape), None, pos))
    refused(lambda: r.rotate(Tensor(shape[0], 4, 64), Tensor(*shape), pos))


@pytest.mark.parametrize("args", [{"head_dim": WRAP + 64}, {"head_dim": 64, "rotary_dim": WRAP + 32},
                                  {"head_dim": 64, "sections": (WRAP + 16, 16)}, {"head_dim": 64, "sections": (-WRAP + 32,)}], ids=str)
def test_shapes_of_heads(args):
    refused(lambda: lib.Rotary(**args))


@pytest.mark.parametrize("rows,vocab", [(WRAP + 3, 100), (3, WRAP + 100), (0, WRAP + 100), (1 << 31, 1)])
def test_logits(rows, vocab):
    refused(lambda: lib.sample(Tensor(rows, vocab), Tensor(rows)))


@pytest.mark.parametrize("how", [{"top_k": 1 << 31}, {"top_k": 1 << 40}, {"top_k": -(1 << 31) - 1}, {"top_k": 50.0}, {"top_k": None},
                                 {"temperature": 10 ** 400}, {"temperature": None}, {"top_p": "0.9"}], ids=str)
def test_settings_of_a_draw(how):
    refused(lambda: lib.sample(Tensor(3, 100), Tensor(3), **how))


def cache():
    return made(lib.KV8Cache, n_layers=2, n_heads=4, n_kv_heads=4, head_dim=64, block_tokens=16, n_blocks=8, max_batch=2, max_blocks=4,
                _ref=None, _scale=0.125)


@pytest.mark.parametrize("name", ["n_layers", "n_heads", "n_kv_heads", "head_dim", "block_tokens", "n_blocks", "max_batch", "max_blocks"])
@pytest.mark.parametrize("off", [WRAP, -WRAP])
def test_shapes_of_a_cache(name, off, monkeypatch):
    for f in ("full", "zeros", "arange"):
        monkeypatch.setattr(torch, f, lambda *a, **k: pytest.fail("allocated"))
    shape = dict(n_layers=2, n_heads=4, n_kv_heads=4, head_dim=64, block_tokens=16, n_blocks=8, max_batch=2, max_blocks=4)
    refused(lambda: lib.KV8Cache(**shape | {name: shape[name] + off}, device="cuda:0"))


def test_steps_of_a_cache(monkeypatch):
    monkeypatch.setattr(torch, "zeros", lambda *a, **k: pytest.fail("allocated"))
    c = cache()
    refused(lambda: c.new_step(1, WRAP + 4))
    refused(lambda: c.new_step(-WRAP + 1, 4))


@pytest.mark.parametrize("layer", [WRAP, -WRAP, WRAP + 1, 2, -1])
def test_layers_of_a_cache(layer):
    """A layer of 2^32 would be layer 0."""
    c, kv = cache(), Tensor(3, 4, 64)
    step = made(lib.KV8Step, cache=c, rows=3, _q=(3, 4, 64), _kv=(3, 4, 64), _slot=1 << 42, _ref=None)
    refused(lambda: c.append(layer, kv, kv, step))
    refused(lambda: c.attention(layer, kv, step))
    refused(lambda: c.read(layer, Tensor(3, dtype=torch.int32)))


def test_slots_to_read():
    refused(lambda: cache().read(0, Tensor(WRAP + 3, dtype=torch.int32)))
