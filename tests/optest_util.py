"""Helpers shared by the tests of the operators around the layers (norm, gated block, distillation loss)."""
import torch

U = 2.0 ** -24                      # half a step of fp32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float8_e4m3fn: 2.0 ** -4}
F64 = torch.float64


def matrix(rows, cols, dtype, pad=0, shift=0, fill=None):
    """rows x cols with rows cols + pad elements apart (pad None: the next multiple of 16 bytes), the first `shift` elements
    past an aligned address.  Whatever lies around the matrix holds `fill` (NaN), for surround_kept."""
    q = 16 // dtype.itemsize
    ld = -(-cols // q) * q if pad is None else cols + pad
    base = torch.full((shift + rows * ld + q,), float("nan") if fill is None else fill, dtype=torch.float32, device="cuda").to(dtype)
    m = torch.as_strided(base, (rows, cols), (ld, 1), shift)
    m.base = base
    return m


def put(values, dtype, **kw):
    m = matrix(values.shape[0], values.shape[1], dtype, **kw)
    m.copy_(values)
    return m


def surround_kept(m):
    """Nothing was written next to the matrix: its buffer holds NaN everywhere else."""
    inside = torch.zeros(m.base.numel(), dtype=torch.bool, device="cuda")
    torch.as_strided(inside, m.shape, m.stride(), m.storage_offset())[:] = True
    return bool(torch.isnan(m.base.float()[~inside]).all())


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def captured(call):
    """The call captured into a graph on a side stream, after one run outside of it; returns the graph."""
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(s.cuda_stream)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call(s.cuda_stream)
    torch.cuda.current_stream().wait_stream(s)
    return g
