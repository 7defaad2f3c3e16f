"""Heads, the cache in 4 bits and attention: what can be checked without a GPU."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import paper_2203_03996_amd as pkg
from paper_2203_03996_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ARGS = {binding.RowsHeadsArgs: "dcnn_rows_heads_args", binding.CacheAppendArgs: "dcnn_cache_append_args", binding.CacheReadArgs: "dcnn_cache_read_args",
        binding.CacheAttendArgs: "dcnn_cache_attend_args"}


def member_of(cls, field):
    """A field of the binding as the header names it."""
    names = [n for n, _ in cls._fields_]
    cache = {"dtype", "heads", "dim", "page", "streams", "length", "num_pages", "codes", "scales", "pages"} if "codes" in names else set()
    if field in cache:
        return "cache." + field + ("_dev" if field in ("codes", "scales", "pages") else "")
    if field in ("rows", "map_rows"):
        return "tokens.list." + field
    if field in ("idx", "count"):
        return f"tokens.list.{field}_dev"
    if field in ("period", "stream", "pos"):
        return "tokens." + field + ("" if field == "period" else "_dev")
    if field in ("table", "positions", "rot", "style"):
        return "rotation." + field + ("_dev" if field == "table" else "")
    norm = re.fullmatch(r"([qk]_norm)_(kind|eps|w|b)", field)
    if norm:
        return f"{norm[1]}.{norm[2]}" + ("_dev" if norm[2] in "wb" else "")
    return field + ("_dev" if field in ("q", "k", "v", "y", "q_out", "k_out", "v_out", "lens", "scratch") else "")


def test_argument_blocks_have_the_layout_of_the_header(tmp_path):
    lines, want = [], []
    for cls, name in ARGS.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(cls))
        for field, _ in cls._fields_:
            if field != "_pad":
                lines.append(f'printf("%zu\\n", offsetof({name}, {member_of(cls, field)}));')
                want.append(getattr(cls, field).offset)
    src = tmp_path / "layout.c"
    src.write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "{ROOT}/include/deltacnn.h"\nint main(void) {{ {" ".join(lines)} return 0; }}\n')
    subprocess.run(["gcc", str(src), "-o", str(tmp_path / "layout")], check=True)
    got = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(v) for v in got] == want


def test_calls_without_a_context_are_refused():
    lib = pkg.load_library()
    for cls, call in ((binding.RowsHeadsArgs, lib.dcnn_rows_heads), (binding.CacheAppendArgs, lib.dcnn_cache_append), (binding.CacheReadArgs, lib.dcnn_cache_read),
                      (binding.CacheAttendArgs, lib.dcnn_cache_attend)):
        assert call(None, C.byref(cls())) == 1


def test_scratch():
    size = pkg.load_library().dcnn_cache_scratch_bytes
    for dtype in range(3):
        sizes = [size(dtype, rows, 8, 8, 64, 4, 4096) for rows in range(0, 9)]
        assert min(sizes) > 0
    for rows, q_heads, heads, dim, streams, length in ((1, 32, 8, 128, 1, 1 << 20), (64, 32, 8, 128, 64, 8192), (5000, 8, 8, 64, 1, 4096), (1, 1, 1, 256, 1, 1 << 30),
                                                       (1 << 15, 1 << 15, 1, 32, 1, 1)):
        assert 0 < size(1, rows, q_heads, heads, dim, streams, length) < 1 << 28
    assert size(0, 0, 1, 1, 32, 1, 1) > 0 and size(3, 1, 8, 8, 64, 1, 64) == 0
    for bad in ((-1, 8, 8, 64, 1, 64), (1, 9, 8, 64, 1, 64), (1, 8, 0, 64, 1, 64), (1, 8, 8, 65, 1, 64), (1, 8, 8, 64, 1, 0), (1, 8, 8, 64, 1, (1 << 30) + 1),
                (1 << 27, 16, 8, 64, 1, 64), (1, 8, 8, 64, 0, 64)):
        assert size(0, *bad) == 0


# ---- the entry points' checks, compiled for the host with launches that count -----------------------------------------
HOST = r"""
#include <cstdarg>
#include "%(src)s/cache.hip"
namespace dcnn {
int launches = 0;
dcnn_status fail(dcnn_ctx* ctx, dcnn_status s, const char* fmt, ...) {
    va_list ap; va_start(ap, fmt); vsnprintf(ctx->err, sizeof(ctx->err), fmt, ap); va_end(ap);
    return s;
}
dcnn_status launch_heads(dcnn_ctx*, int, int, HeadsOp, const HeadsArgs&) { ++launches; return DCNN_OK; }
dcnn_status launch_attend(dcnn_ctx*, int, int, const AttendPlan&, const AttendArgs&) { ++launches; return DCNN_OK; }
AttendPlan attend_plan(int, int64_t, int, int, int, int64_t, int64_t) { return AttendPlan(); }
}
extern "C" {
dcnn_ctx ctx_of_tests;
dcnn_ctx* test_ctx() { return &ctx_of_tests; }
const char* test_error() { return ctx_of_tests.err; }
int test_launches() { int n = launches; launches = 0; return n; }
}
"""


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    at = tmp_path_factory.mktemp("host")
    (at / "host.cpp").write_text(HOST % {"src": os.path.join(ROOT, "paper_2203_03996_amd", "csrc")})
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-w", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-o", str(at / "host.so"), str(at / "host.cpp")], check=True)
    lib = C.CDLL(str(at / "host.so"))
    lib.test_ctx.restype = C.c_void_p
    lib.test_error.restype = C.c_char_p
    for cls, name in ARGS.items():
        getattr(lib, name[:-5]).argtypes = [C.c_void_p, C.POINTER(cls)]
    return lib


BASE = 1 << 20                                      # (addresses that nothing reads)


def fill(a, **over):
    """Arguments of a call that is taken: 4 rows, 2 heads of 64, everything apart."""
    names = [n for n, _ in a._fields_]
    good = dict(rows=4, map_rows=4, period=64, dtype=1, heads=2, dim=64, page=16, streams=2, length=64, num_pages=8, codes=BASE, scales=2 * BASE, pages=3 * BASE,
                q=4 * BASE, k=5 * BASE, v=6 * BASE, y=7 * BASE, q_out=8 * BASE, k_out=9 * BASE, v_out=10 * BASE, q_heads=4, k_heads=2, ldq=256, ldk=128, ldv=128, ldy=256,
                ldq_out=256, ldk_out=128, scale=0.125, table=11 * BASE, positions=64, rot=64, style=0, lens=12 * BASE, scratch=13 * BASE, scratch_bytes=1 << 19,
                q_norm_kind=1, q_norm_eps=1e-5, k_norm_kind=2, k_norm_eps=1e-5)
    for name, value in {**good, **over}.items():
        if name in names:
            setattr(a, name, value)
    return a


CALLS = {"heads": (binding.RowsHeadsArgs, "dcnn_rows_heads"), "append": (binding.CacheAppendArgs, "dcnn_cache_append"), "read": (binding.CacheReadArgs, "dcnn_cache_read"),
         "attend": (binding.CacheAttendArgs, "dcnn_cache_attend")}
EVERY = dict(rows=[-1, 1 << 31, 5], map_rows=[-1, 1 << 31], idx=[BASE + 2], count=[BASE + 1], pos=[BASE + 2])
CACHE = dict(dtype=[3, -1, 7], heads=[0, -2, 65537], dim=[0, 48, 160, 512], page=[0, 8, 17, 8192], streams=[0, -1, 1 << 31], length=[0, (1 << 30) + 1, -5],
             num_pages=[0, 1 << 31], codes=[0, BASE + 8], scales=[0, BASE * 2 + 4], pages=[BASE * 3 + 1], stream=[BASE + 3], period=[0, -1, 1 << 31])
NORM = {k + "_" + n: v for k in ("k_norm",) for n, v in dict(kind=[-1, 3], eps=[-1.0, float("nan"), float("inf")], w=[BASE + 1], b=[BASE + 1]).items()}
ROTATION = dict(positions=[0, -1, 1 << 31], rot=[0, 8, 24, 80], style=[-1, 2], table=[11 * BASE + 4])
WRONG = {
    "heads": dict(EVERY, **NORM, **ROTATION, dtype=[3], dim=[40], q_heads=[0, 65537], k_heads=[-1], q=[0, BASE + 1], k=[0], q_out=[0], k_out=[0, 8 * BASE + 2], ldq=[255, 1 << 31],
                  ldk=[127], ldq_out=[10], ldk_out=[10], q_norm_kind=[5], period=[0]),
    "append": dict(EVERY, **CACHE, **NORM, **ROTATION, k=[0, BASE, 5 * BASE + 1], v=[0, 2 * BASE], ldk=[127], ldv=[0]),
    "read": dict(EVERY, **CACHE, k_out=[BASE + 64, 10 * BASE + 2, 9 * BASE + 1], ldk=[100], ldv=[100]),
    "attend": dict(EVERY, **CACHE, q_heads=[0, 3, 65538], q=[0], y=[0, 4 * BASE + 2, BASE, 13 * BASE], ldq=[255], ldy=[-1], scale=[float("nan"), float("inf")], window=[-1],
                   lens=[BASE + 2], scratch=[0, BASE + 8], scratch_bytes=[0]),
}


@pytest.mark.parametrize("call", list(CALLS))
def test_refusals(host, call):
    cls, name = CALLS[call]
    run = getattr(host, name)
    ctx = host.test_ctx()
    extra = dict(causal=1) if call == "attend" else {}
    assert run(ctx, fill(cls(), **extra)) == 0 and host.test_launches() == 1, host.test_error()
    assert run(ctx, fill(cls(), rows=0, **extra)) == 0 and host.test_launches() == 0
    for field, values in WRONG[call].items():
        for v in values:
            status = run(ctx, fill(cls(), **{**extra, field: v}))
            assert status != 0 and host.test_launches() == 0, f"{call}: {field} = {v} was taken"
            assert host.test_error(), f"{call}: {field} = {v}"
    assert run(ctx, fill(cls(), idx=14 * BASE, count=14 * BASE, stream=14 * BASE, pos=14 * BASE, period=0, **extra)) == 0 and host.test_launches() == 1
    if call == "read":
        assert run(ctx, fill(cls(), k_out=0, v_out=0)) != 0
        assert run(ctx, fill(cls(), k_out=0)) == 0 and run(ctx, fill(cls(), v_out=0)) == 0 and host.test_launches() == 2
    else:
        big = dict(rows=1 << 29, map_rows=1 << 29, heads=8, q_heads=8, k_heads=8, ldq=512, ldk=512, ldv=512, ldy=512, ldq_out=512, ldk_out=512)
        assert run(ctx, fill(cls(), **{**big, **extra})) == 7 and host.test_launches() == 0
    if call != "heads":
        assert run(ctx, fill(cls(), pages=0, num_pages=7)) != 0 and host.test_launches() == 0
        assert run(ctx, fill(cls(), heads=65536, q_heads=65536, page=4096, dim=256)) == 7


def test_in_place_heads(host):
    ctx, cls = host.test_ctx(), binding.RowsHeadsArgs
    assert host.dcnn_rows_heads(ctx, fill(cls(), q_out=4 * BASE, k_out=5 * BASE)) == 0
    assert host.dcnn_rows_heads(ctx, fill(cls(), q_out=4 * BASE, ldq_out=512)) != 0
    assert host.dcnn_rows_heads(ctx, fill(cls(), q_out=4 * BASE + 256)) != 0
    assert host.dcnn_rows_heads(ctx, fill(cls(), q_out=5 * BASE)) != 0          # q's output over k
    assert host.dcnn_rows_heads(ctx, fill(cls(), k_heads=0, k=0, k_out=0)) == 0
    # queries and keys as columns of one matrix
    assert host.dcnn_rows_heads(ctx, fill(cls(), k=4 * BASE + 512, ldq=384, ldk=384, q_out=4 * BASE, ldq_out=384, k_out=4 * BASE + 512, ldk_out=384)) == 0


# ---- the binding, with CPU tensors in the place of the GPU's ----------------------------------------------------------
class Lib:
    """Takes every call down."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda handle, a=None, *rest: self.calls.append((name, a)) or 0

    def dcnn_cache_scratch_bytes(self, *sizes):
        return 256


@pytest.fixture
def ctx():
    c = pkg.Context.__new__(pkg.Context)
    c.lib, c.index, c.stream, c.handle, c._gpu = Lib(), -1, None, None, torch.device("cpu")
    c.empty = lambda shape, dtype: torch.empty(shape, dtype=dtype)
    c.capturing = lambda: False
    return c


def cache_of(ctx, **kw):
    kw = {**dict(streams=2, length=40, heads=2, dim=64, page=16), **kw}
    codes = kw.pop("codes", torch.zeros(6, 2, 2, 16, 32, dtype=torch.uint8))
    scales = kw.pop("scales", torch.zeros(6, 2, 2, 16, 2, dtype=torch.uint8))
    return pkg.TokenCache(ctx, kw.pop("streams"), kw.pop("length"), kw.pop("heads"), kw.pop("dim"), codes=codes, scales=scales, **kw)


def half(*shape):
    return torch.zeros(*shape, dtype=torch.float16)


def int32(*v):
    return torch.tensor(v, dtype=torch.int32)


def test_caches_that_do_not_fit_are_refused(ctx):
    cache_of(ctx)
    u8 = torch.uint8
    for wrong in (dict(dtype=torch.float64), dict(page=24), dict(page=8), dict(dim=48), dict(streams=3), dict(streams=0), dict(heads=3), dict(length=49), dict(num_pages=5),
                  dict(codes=torch.zeros(6, 2, 2, 16, 32)), dict(codes=torch.zeros(6, 2, 2, 16, 64, dtype=u8)[..., ::2]), dict(scales=torch.zeros(5, 2, 2, 16, 2, dtype=u8)), dict(scales=None),
                  dict(pages=torch.zeros(2, 2, dtype=torch.int32)), dict(pages=torch.zeros(2, 3)), dict(pages=torch.zeros(3, 2, dtype=torch.int32).T)):
        with pytest.raises(ValueError):
            cache_of(ctx, **wrong)
    assert cache_of(ctx, streams=5, pages=torch.zeros(5, 3, dtype=torch.int32)).num_pages == 6          # (pages may be shared)


def test_rotations_that_do_not_fit_are_refused():
    table = torch.zeros(10, 16, 2)
    assert pkg.Rotation(table).rot == 32 and pkg.Rotation(table, "pairs").style == 1
    for wrong in (torch.zeros(10, 12, 2), torch.zeros(10, 16), torch.zeros(10, 16, 2, dtype=torch.float16), torch.zeros(0, 16, 2), torch.zeros(10, 2, 16).transpose(1, 2)):
        with pytest.raises(ValueError):
            pkg.Rotation(wrong)
    with pytest.raises(KeyError):
        pkg.Rotation(table, "thirds")
    with pytest.raises(ValueError):
        pkg.Rotation(table).pointers(0)
    r = pkg.Rotation.of_positions(100, 32, device="cpu")
    angle = 99.0 * 10000.0 ** (-torch.arange(16, dtype=torch.float64) / 16)
    assert torch.allclose(r.table[99].double(), torch.stack([angle.cos(), angle.sin()], 1), rtol=0, atol=2.0 ** -24)


def test_which_tokens_a_call_names(ctx):
    """Period, arrays and room of the rows, as the entry points get them."""
    cache, q = cache_of(ctx), half(3, 256)
    seen = ctx.lib.calls
    cache.attend(q)
    assert (seen[-1][1].rows, seen[-1][1].map_rows, seen[-1][1].period, seen[-1][1].q_heads) == (3, 3, 40, 4)
    cache.attend(q, positions=int32(1, 2, 3, 4))
    assert (seen[-1][1].rows, seen[-1][1].map_rows, seen[-1][1].period) == (3, 4, 1)
    idx = int32(0, 70, 79)
    cache.attend(q, idx=idx)
    assert (seen[-1][1].rows, seen[-1][1].period, seen[-1][1].idx) == (3, 40, idx.data_ptr()) and seen[-1][1].map_rows >= 80
    cache.attend(q, idx=int32(1, 0), count=int32(1), streams=int32(0, 1), positions=int32(3, 4))
    assert (seen[-1][1].rows, seen[-1][1].map_rows) == (2, 2)
    assert cache.attend(half(5, 256), idx=int32(*range(9)), count=int32(2)).shape == (5, 256)       # (room for five of nine)
    cache.append(half(3, 128), half(3, 128), streams=int32(0, 1, 1), positions=int32(0, 0, 1))
    assert [t.shape for t in cache.read(positions=int32(1, 2))] == [(2, 128)] * 2 and cache.read()[0].shape == (80, 128)
    rotation = pkg.Rotation(torch.zeros(40, 32, 2))
    ctx.rows_heads(half(3, 256), half(3, 128), dim=64, rotation=rotation)
    assert (seen[-1][1].q_heads, seen[-1][1].k_heads, seen[-1][1].period, seen[-1][1].positions) == (4, 2, 40, 40)


def test_tensors_that_do_not_fit_are_refused(ctx):
    cache, rotation = cache_of(ctx), pkg.Rotation(torch.zeros(40, 32, 2))
    idx, count = int32(0, 1, 2, 3), int32(2)
    wrong = [
        lambda: cache.attend(half(3, 250)), lambda: cache.attend(half(3, 256).float()), lambda: cache.attend(half(256, 3).T), lambda: cache.attend(half(3, 4, 64)),
        lambda: cache.attend(half(3, 256), idx=idx), lambda: cache.attend(half(3, 256), positions=int32(1, 2)), lambda: cache.attend(half(3, 256), streams=int32(0, 0, 0)),
        lambda: cache.attend(half(3, 256), positions=torch.zeros(3)), lambda: cache.attend(half(3, 256), lens=int32(1)), lambda: cache.attend(half(3, 256), out=half(2, 256)),
        lambda: cache.attend(half(3, 256), out=half(3, 128)), lambda: cache.attend(half(3, 256), idx=idx.long(), count=count),
        lambda: cache.append(half(3, 128), half(2, 128)), lambda: cache.append(half(3, 256), half(3, 256)), lambda: cache.append(half(3, 128), half(3, 128), norm=pkg.RowNorm("rms", half(128))),
        lambda: ctx.rows_heads(half(3, 256), half(2, 128), dim=64), lambda: ctx.rows_heads(half(3, 256), half(3, 128).float(), dim=64), lambda: ctx.rows_heads(half(3, 250), dim=64),
        lambda: ctx.rows_heads(half(3, 256), dim=64, rotation=rotation, positions=int32(1)), lambda: ctx.rows_heads(half(3, 256), dim=64, q_out=half(3, 128)),
        lambda: ctx.rows_heads(half(3, 256), dim=64, idx=idx), lambda: ctx.rows_heads(torch.zeros(3, 256, dtype=torch.float64), dim=64),
    ]
    for i, call in enumerate(wrong):
        before = len(ctx.lib.calls)
        with pytest.raises(ValueError):
            call()
        assert len(ctx.lib.calls) == before, i
