"""Inputs and layouts shared by the tests of the token operators."""
import torch

from paper_2609_36246_amd import _lib as L

BF16, F32 = torch.bfloat16, torch.float32
U32, U16 = 2.0 ** -24, 2.0 ** -8      # unit roundoffs of fp32 and bf16 (8-bit significand)


def unit(dtype):
    return U16 if dtype == BF16 else U32


def kind(dtype):
    return L.OLIVE_BF16 if dtype == BF16 else L.OLIVE_F32


def f64(t):
    return t.detach().double().cpu().numpy()


def matrix(rows, width, dtype, how="plain", gen=None, std=1.0, mean=0.0, fill=float("nan")):
    """A [rows, width] matrix, of normal values with `gen`, else of `fill`, in one of several
    layouts: "plain"; "part", columns of longer rows; "odd", at an address and a row distance
    that are not multiples of anything."""
    if how == "plain":
        x = torch.full((rows, width), fill, dtype=dtype, device="cuda")
    elif how == "part":
        x = torch.full((rows, width + 24), fill, dtype=dtype, device="cuda")[:, 8:8 + width]
    else:
        flat = torch.full((rows * (width + 3) + 1,), fill, dtype=dtype, device="cuda")
        x = flat[1:].as_strided((rows, width), (width + 3, 1))
    if gen is not None:
        x.copy_((torch.randn(rows, width, generator=gen) * std + mean).to(dtype))
    return x


def graph_of(call):
    """A graph of `call`, made on a stream of its own after a first run there."""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        call()
    torch.cuda.synchronize()
    return g
