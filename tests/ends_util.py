"""Helpers of the tests of a word model's ends."""
EPS = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
# half a step below the smallest normal number
TINY = {"float32": 2.0 ** -150, "bfloat16": 2.0 ** -134, "float16": 2.0 ** -25}


def dtype_of(name):
    import torch
    return getattr(torch, name)


def generator(seed):
    import torch
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def matrix(g, rows, cols, name, scale=1.0, pad=0):
    """rows x cols of normal values inside a wider buffer of NaN, so that a read
    past a row's end shows."""
    import torch
    buf = torch.full((rows, cols + pad), float("nan"), dtype=dtype_of(name))
    buf[:, :cols] = (torch.randn((rows, cols), generator=g) * scale).to(buf.dtype)
    return buf.cuda()[:, :cols]


def guarded(rows, cols, name, pad=3, fill=7.0):
    """An output of rows x cols inside a wider buffer, and a check that nothing
    else of it was written."""
    import torch
    buf = torch.full((rows + 2, cols + pad), fill, dtype=dtype_of(name), device="cuda")
    view = buf[1:rows + 1, :cols]

    def untouched():
        left = buf.clone()
        left[1:rows + 1, :cols] = fill
        return bool((left == fill).all())

    return view, untouched


def captured(call):
    """A graph of call() (run once before on another stream), and what it
    returned."""
    import torch
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    return graph, out
