"""Row operators: what can be checked without a GPU."""
import ctypes as C

import pytest

import paper_2203_03996_amd as pkg
from paper_2203_03996_amd.binding import RowsMatmulArgs, RowsNormArgs


def test_sizes_of_packed_weights_and_scratch():
    lib = pkg.load_library()
    size = lib.dcnn_rows_weights_bytes
    for k, n in ((1, 1), (64, 33), (128, 32), (129, 32), (4096, 4096), (65536, 100)):
        need = -(-k // 128) * 128 * (-(-n // 32) * 32) + -(-n // 32) * 32 * 4      # 8-bit weights in whole blocks, a scale per channel
        assert need <= size(k, n) < need + 256 and size(k, n) % 256 == 0
    for k, n in ((0, 4), (4, 0), (-1, 4), (65537, 4), (4, (1 << 24) + 1)):
        assert size(k, n) == 0 and lib.dcnn_rows_scratch_bytes(4, k, n, 1) == 0
    for rows, k in ((0, 64), (1, 1), (7, 65), (1000, 4096)):
        assert lib.dcnn_rows_scratch_bytes(rows, k, 64, 1) >= rows * (k + 4) + lib.dcnn_rows_scratch_bytes(rows, k, 64, 0)
        assert lib.dcnn_rows_scratch_bytes(rows, k, 64, 0) < 16 << 20          # (counts and partial sums)
    assert lib.dcnn_rows_scratch_bytes(-1, 64, 64, 0) == 0


def test_scratch_grows_with_the_rows():
    """Scratch of some rows is enough for every call with fewer of them."""
    lib = pkg.load_library()
    rows = sorted({int(2 ** (i / 8)) + d for i in range(8, 137) for d in (-1, 0, 1)})
    for k, n in ((64, 64), (2048, 256), (4096, 512), (4096, 4096), (8192, 1024), (16384, 8192), (65536, 64), (8192, 16384), (8192, 16385)):
        for linear in (0, 1):
            sizes = [lib.dcnn_rows_scratch_bytes(r, k, n, linear) for r in rows]
            assert sizes == sorted(sizes), (k, n, linear)
        assert lib.dcnn_rows_scratch_bytes(rows[-1], k, n, 0) < 16 << 20


def test_calls_without_a_context_are_refused():
    lib = pkg.load_library()
    assert lib.dcnn_rows_norm(None, C.byref(RowsNormArgs())) == 1
    assert lib.dcnn_rows_matmul(None, C.byref(RowsMatmulArgs())) == 1 and lib.dcnn_rows_linear(None, C.byref(RowsMatmulArgs())) == 1
    assert lib.dcnn_rows_pack(None, 0, 4, 4, None, 4, None, None, 0) == 1


def test_layers_and_networks_keep_to_their_types():
    """The types that only row operators take."""
    from paper_2203_03996_amd.binding import LayerSizes
    lib = pkg.load_library()
    for dtype in (pkg.BF16, pkg.I8):
        desc = pkg.make_desc(pkg.ACT, dtype, 2, 16, 16, 64, act=pkg.ACT_RELU)
        assert lib.dcnn_layer_query(C.byref(desc), C.byref(LayerSizes())) == 3


def test_norm_kinds():
    assert pkg.RowNorm("rms").kind == 1 and pkg.RowNorm("layer").kind == 2 and pkg.RowNorm("none").kind == 0
    with pytest.raises(KeyError):
        pkg.RowNorm("batch")


def test_argument_blocks_have_the_layout_of_the_header(tmp_path):
    """The binding spells nested members out: sizes and offsets against a C compiler's."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = {RowsNormArgs: "dcnn_rows_norm_args", RowsMatmulArgs: "dcnn_rows_matmul_args"}
    plain = {"post": "post.", "pre": "pre."}
    lines, want = [], []
    for cls, name in names.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(cls))
        for field, _ in cls._fields_:
            if field == "_pad":
                continue
            first = field.split("_")[0]
            member = field
            if field in ("rows", "map_rows"):
                member = "list." + field
            elif field in ("idx", "count"):
                member = f"list.{field}_dev"
            elif first in plain and field != first:
                rest = field[len(first) + 1:]
                member = plain[first] + (rest + "_dev" if rest in ("w", "b") else rest)
            elif getattr(cls, field).size == 8 and field in ("x", "h", "gate", "y", "z", "q", "q_scale", "packed", "bias", "scratch"):
                member = field + "_dev"
            lines.append(f'printf("%zu\\n", offsetof({name}, {member}));')
            want.append(getattr(cls, field).offset)
    src = tmp_path / "layout.c"
    src.write_text(f'#include <stdio.h>\n#include "{root}/include/deltacnn.h"\nint main(void) {{ {" ".join(lines)} return 0; }}\n')
    subprocess.run(["gcc", str(src), "-o", str(tmp_path / "layout")], check=True)
    got = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(v) for v in got] == want


@pytest.mark.parametrize("move", ["half", "half and back", "data", "to"])
def test_a_norm_reads_its_parameters_where_they_lie_at_each_call(move):
    """A module's parameters keep their tensors and change what these stand on; the address of a call is the one of that moment."""
    import torch
    layer = torch.nn.LayerNorm(64)
    norm = pkg.RowNorm("layer", layer.weight, layer.bias)
    assert norm.pointers(64, torch.float32, -1) == (2, norm.eps, layer.weight.data_ptr(), layer.bias.data_ptr())
    dtype = torch.float32
    held = layer.weight.data, layer.bias.data                     # (so that the new storage is not the old one's by chance)
    if move == "half":
        layer.half()
        dtype = torch.float16
    elif move == "half and back":
        layer.half().float()
    elif move == "to":
        layer.to(torch.bfloat16)
        dtype = torch.bfloat16
    else:
        layer.weight.data, layer.bias.data = torch.ones(64), torch.zeros(64)
    assert norm.pointers(64, dtype, -1)[2:] == (layer.weight.data_ptr(), layer.bias.data_ptr())
    assert layer.weight.data_ptr() != held[0].data_ptr()
    for wrong in (t for t in (torch.float32, torch.float16, torch.bfloat16) if t != dtype):
        with pytest.raises(ValueError):
            norm.pointers(64, wrong, -1)
    layer.bias.data = torch.zeros(65, dtype=dtype)
    with pytest.raises(ValueError):
        norm.pointers(64, dtype, -1)
    layer.bias.data = torch.zeros(128, dtype=dtype)[::2]
    with pytest.raises(ValueError):
        norm.pointers(64, dtype, -1)


def test_scratch_that_a_graph_clears_is_not_kept(monkeypatch):
    """What is captured on the context's stream decides, not the stream that torch is on (streams and captures are stood in for)."""
    import contextlib

    import torch
    current, captured = ["torch's"], set()

    @contextlib.contextmanager
    def on(stream):
        before, current[0] = current[0], stream
        yield
        current[0] = before
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: current[0] in captured)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: current[0], raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    ctx = pkg.Context.__new__(pkg.Context)
    ctx.lib, ctx.index, ctx.stream, ctx._raw_stream, ctx._gpu = pkg.load_library(), 0, "the context's", "the context's", torch.device("cpu")
    weights = pkg.RowWeights.__new__(pkg.RowWeights)
    weights.__dict__.update(ctx=ctx, k=64, n=64, _grown=None, _grown_rows=0, _captured=set())
    captured.add("the context's")
    weights._linear_scratch(100)                                   # torch is on another stream, which no graph captures
    assert weights._grown is None
    captured.clear()
    captured.add("torch's")
    weights._linear_scratch(100)                                   # the other way round: the scratch is cleared now
    assert weights._grown is not None and not weights._captured
    captured.add("the context's")
    at, _ = weights._linear_scratch(100)                           # a graph that uses it holds it
    assert at == weights._grown.data_ptr() and len(weights._captured) == 1


def test_new_tensors_and_captures_are_those_of_the_contexts_gpu(monkeypatch):
    """Two GPUs whose streams have the same handle (the default one, 0), and torch is on the other (both are stood in for)."""
    import contextlib

    import torch
    made, entered = [], []

    @contextlib.contextmanager
    def on(stream):
        entered.append(stream)
        yield
    monkeypatch.setattr(torch, "empty", lambda shape, dtype, device: made.append(device))
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: bool(entered))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    ctx = pkg.Context.__new__(pkg.Context)
    ctx.device, ctx._gpu, ctx.index, ctx.stream, ctx._raw_stream = torch.device("cuda"), torch.device("cuda", 0), 0, "the context's", 0
    ctx.empty((3, 4), torch.float32)
    assert made == [torch.device("cuda", 0)]
    assert ctx.capturing() and entered == ["the context's"]        # asked of the context's stream, not of the other GPU's


def test_threads_take_turns_at_the_scratch_of_a_product(monkeypatch):
    """A call is two launches that share scratch: no other call may come between its choice of scratch and its last launch (the library stood in for)."""
    import threading
    import time

    import torch
    inside, together, used = [], [], []

    def call(handle, a):
        inside.append(a)
        time.sleep(0.002)                                          # (the interpreter's lock is not held in the library either)
        together.append(len(inside))
        used.append((a.rows, a.scratch_bytes))
        inside.remove(a)
        return 0

    class Row(pkg.binding.RowsMatmulArgs):
        __hash__ = object.__hash__
    weights = pkg.RowWeights.__new__(pkg.RowWeights)
    ctx = pkg.Context.__new__(pkg.Context)
    ctx.lib, ctx.index, ctx.handle, ctx._gpu, ctx.stream = pkg.load_library(), -1, None, torch.device("cpu"), None
    monkeypatch.setattr(ctx, "empty", lambda shape, dtype: torch.empty(shape, dtype=dtype), raising=False)
    monkeypatch.setattr(ctx, "capturing", lambda: False, raising=False)
    weights.__dict__.update(ctx=ctx, k=64, n=64, bias=None, act=0, packed=torch.zeros(1), _grown=None, _grown_rows=0, _captured=set(), _scratch_at=(0, 0),
                            _one_call=threading.Lock())
    threads = [threading.Thread(target=lambda r=r: [weights._call(call, 1, Row(), r, torch.float16, None, None) for _ in range(5)]) for r in (70, 200, 500, 900)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(used) == 20 and set(together) == {1}
    assert all(size >= ctx.lib.dcnn_rows_scratch_bytes(rows, 64, 64, 1) for rows, size in used)
