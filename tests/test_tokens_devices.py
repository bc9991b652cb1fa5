"""Tensors that a token operator's descriptor holds and that are not on the current device: refused
before the library is entered, which would follow their addresses (no GPU needed)."""
import pytest
import torch

from paper_2609_36246_amd import _lib as L

BF16, I32 = torch.bfloat16, torch.int32
HERE = 3


class Here(torch.Tensor):
    def get_device(self):
        return HERE


class Elsewhere(torch.Tensor):
    def get_device(self):
        return 1


def here(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Here)


PLACES = {"another GPU": lambda t: t.as_subclass(Elsewhere), "the CPU": lambda t: t}
X, TOK = here(6, 64, dtype=BF16), here(6, dtype=I32)
FIELDS = {"ids": (6, I32), "weight": (64, BF16), "bias": (64, BF16), "uniform": (6, torch.float32),
          "temperature": (6, torch.float32), "top_k": (6, I32), "top_p": (6, torch.float32), "min_p": (6, torch.float32)}


def embed(**t):
    d = L.make_embed_desc(6, 6, 64, t["ids"])
    return [lambda: L.olive_embed(d, X, X, stream=0), lambda: L.olive_embed_backward(d, X, X, stream=0)]


def norm(**t):
    d = L.make_norm_desc(6, 64, t.get("weight"), t.get("bias"))
    return [lambda: L.olive_row_norm(d, X, X, stream=0), lambda: L.olive_row_norm_backward(d, X, X, X, stream=0)]


def sample(**t):
    d = L.make_sample_desc(6, 64, **{"uniform": here(6), **t})
    return [lambda: L.olive_sample(d, X, TOK, stream=0)]


OPERATORS = {"ids": embed, "weight": norm, "bias": norm, "uniform": sample, "temperature": sample, "top_k": sample,
             "top_p": sample, "min_p": sample}


@pytest.fixture
def entered(monkeypatch):
    calls = []
    monkeypatch.setattr(L, "_call", lambda name: lambda *a: calls.append(name) or 0)
    monkeypatch.setattr(L, "_here", lambda: HERE)
    return calls


@pytest.mark.parametrize("place", PLACES)
@pytest.mark.parametrize("field", FIELDS)
def test_one_tensor_elsewhere(field, place, entered):
    n, dtype = FIELDS[field]
    for call in OPERATORS[field](**{field: here(n, dtype=dtype)}):
        call()
    assert entered
    del entered[:]
    try:
        calls = OPERATORS[field](**{field: PLACES[place](torch.zeros(n, dtype=dtype))})
    except ValueError as e:             # (with others that are here)
        assert "on devices" in str(e)
        calls = []
    for call in calls:
        with pytest.raises(ValueError, match="on device -?1, and the current one is 3"):
            call()
    assert not entered


def test_tensors_of_two_devices(entered):
    with pytest.raises(ValueError, match="on devices"):
        L.make_norm_desc(6, 64, here(64, dtype=BF16), torch.zeros(64, dtype=BF16))
    with pytest.raises(ValueError, match="on devices"):
        L.make_sample_desc(6, 64, here(6), min_p=torch.zeros(6).as_subclass(Elsewhere))


def test_what_is_not_read_may_be_anywhere(entered):
    """No tokens or rows: nothing that the descriptor holds is read. Addresses are the caller's."""
    none = here(0, 64, dtype=BF16)
    L.olive_embed(L.make_embed_desc(0, 6, 64, torch.zeros(0, dtype=I32)), X, none, stream=0)
    L.olive_row_norm(L.make_norm_desc(0, 64, torch.zeros(64, dtype=BF16)), none, none, stream=0)
    L.olive_sample(L.make_sample_desc(0, 64, torch.zeros(0)), none, here(0, dtype=I32), stream=0)
    L.olive_row_norm(L.make_norm_desc(6, 64, 1 << 20), X, X, stream=0)
    assert len(entered) == 4
