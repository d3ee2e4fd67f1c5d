"""The token operators' host side without a GPU: what the calls refuse, workspace sizes, struct layouts.

A call checks its arguments before it touches the device, so a context that is all zeros (no stream, no
workspace) and addresses that nothing reads are enough."""
import ctypes as C
import os
import re
import subprocess

import pytest

import paper_2608_27735_gb300 as ab

F16, F32, BF16 = ab.ABCD_F16, ab.ABCD_F32, ab.ABCD_BF16
OK, BAD, WORKSPACE = ab.ABCD_OK, ab.ABCD_ERR_INVALID_ARG, ab.ABCD_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    ab.build()
    return ab.lib()


@pytest.fixture
def ctx():
    return C.create_string_buffer(1 << 16)


BASE = 1 << 40


def matrix(rows, cols, at=0, dtype=BF16, stride=None):
    """A matrix `at` MiB (or bytes past them, by fractions) behind BASE."""
    return ab.abcd_matrix(BASE + int(at * (1 << 20)), rows, cols, stride or cols, dtype)


def ref(m):
    return None if m is None else C.byref(m)


def address(at):
    return BASE + int(at * (1 << 20))


def last(lib, ctx):
    return lib.abcd_last_error(ctx).decode()


class Call:
    """A call with arguments by name; `with_` replaces some."""

    def __init__(self, function, **args):
        self.function, self.args = function, args

    def __call__(self, ctx, **changed):
        assert set(changed) <= set(self.args)
        return self.function(ctx, *[ref(v) if isinstance(v, C.Structure) else v for v in {**self.args, **changed}.values()])


def test_struct_layouts(tmp_path):
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    structs = {"abcd_matrix": ab.abcd_matrix, "abcd_norm": ab.abcd_norm, "abcd_packed8": ab.abcd_packed8}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "abcd.h"', "int main(void){"]
    for name, py in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));' for f, _ in py._fields_]
    src.write_text("\n".join(lines + ["return 0;}"]))
    subprocess.run(["gcc", "-I", os.path.dirname(ab.HEADER), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    got = dict(l.rsplit(" ", 1) for l in out.strip().splitlines())
    from paper_2608_27735_gb300 import network
    for name, py in structs.items():
        assert int(got[name]) == C.sizeof(py)
        for f, _ in py._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(py, f).offset
    # the same as bytes
    n = ab.abcd_norm.from_buffer_copy(network._pack_norm(1, 16, 32, 0.5, 48, 64).ljust(C.sizeof(ab.abcd_norm)))
    assert (n.kind, n.weight, n.bias, n.eps, n.mean, n.rstd) == (1, 16, 32, 0.5, 48, 64)
    q = ab.abcd_packed8.from_buffer_copy(network._pack_packed(16, 32, 3, 40, 64, 2))
    assert (q.codes, q.powers, q.rows, q.cols, q.stride, q.power_stride) == (16, 32, 3, 40, 64, 2)


def test_constants_are_the_headers():
    text = open(ab.HEADER).read()
    for name in ("ABCD_I32", "ABCD_I64", "ABCD_NO_ACTIVATION", "ABCD_LAYER_NORM", "ABCD_RMS_NORM"):
        assert int(re.search(name + r" = (\d+)", text)[1]) == getattr(ab, name)


def test_workspace_sizes(lib):
    size = C.c_size_t()
    def of(call, *args):
        assert getattr(lib, call)(*args, C.byref(size)) == OK, (call, args)
        return size.value
    assert of("abcd_embedding_workspace_size", 0, 1, 1) >= 65536
    assert of("abcd_embedding_workspace_size", 1 << 30, 1 << 30, 16) > 16 << 30
    assert of("abcd_linear_workspace_size", 100, 64, 64, F32) > of("abcd_linear_workspace_size", 100, 64, 64, BF16)
    assert of("abcd_residual_norm_workspace_size", 10, 64) < of("abcd_residual_norm_workspace_size", 1000, 64)
    assert of("abcd_packed8_workspace_size", 100, 64, 256, F32) > of("abcd_network_workspace_size", 100, 64, 256, F32)
    for call, args in (("abcd_embedding_workspace_size", (-1, 1, 1)), ("abcd_embedding_workspace_size", (1, 0, 1)),
                       ("abcd_embedding_workspace_size", (1, 1, 0)), ("abcd_linear_workspace_size", (1, 1, 0, F32)),
                       ("abcd_linear_workspace_size", (1, 1, 1, 7)), ("abcd_residual_norm_workspace_size", (1, 0)),
                       ("abcd_packed8_workspace_size", (1, 1, 0, F32))):
        assert getattr(lib, call)(*args, C.byref(size)) == BAD
        assert getattr(lib, call)(*args, None) == BAD


def test_embedding_refusals(lib, ctx):
    call = Call(lib.abcd_embedding, table=matrix(100, 64), index=address(1), kind=ab.ABCD_I64, scale=1.0, add=matrix(8, 64, 2), y=matrix(8, 64, 3))
    assert call(ctx) == WORKSPACE                    # all that is missing
    table, y = matrix(100, 64), matrix(8, 64, 3)
    for change in (dict(table=matrix(100, 63)), dict(table=matrix(0, 64)), dict(table=matrix(100, 64, dtype=F32)),
                   dict(table=matrix(100, 64, 1e-6)), dict(index=None), dict(index=address(1) + 4), dict(kind=0),
                   dict(kind=ab.ABCD_I32, index=address(1) + 2), dict(scale=float("inf")), dict(scale=float("nan")),
                   dict(add=matrix(9, 64, 2)), dict(add=matrix(8, 64, 2, F16)), dict(y=None), dict(table=None)):
        assert call(ctx, **change) == BAD, change
    assert lib.abcd_embedding(None, ref(table), address(1), ab.ABCD_I64, 1.0, None, ref(y)) == BAD
    back = Call(lib.abcd_embedding_backward, dy=matrix(8, 64, 3), index=address(1), kind=ab.ABCD_I32, scale=1.0, dtable=matrix(100, 64))
    assert back(ctx) == WORKSPACE
    for change in (dict(dtable=matrix(100, 65)), dict(dtable=matrix(0, 64)), dict(dtable=matrix(100, 64, 3)), dict(dtable=matrix(100, 64, 1)),
                   dict(scale=float("nan")), dict(index=None), dict(dy=matrix(8, 64, 3, F32)), dict(kind=5)):
        assert back(ctx, **change) == BAD, change


def test_linear_refusals(lib, ctx):
    call = Call(lib.abcd_linear, x=matrix(20, 64), weight=matrix(48, 64, 1), bias=address(2), bias_dtype=F32, act=ab.ABCD_GELU,
                residual=matrix(20, 48, 3), y=matrix(20, 48, 4), z=matrix(20, 48, 5))
    assert call(ctx) == WORKSPACE
    assert call(ctx, y=matrix(20, 48, 3)) == WORKSPACE              # over the residual
    for change in (dict(x=matrix(20, 63)), dict(weight=matrix(48, 65, 1)), dict(weight=matrix(48, 64, 1, F16)), dict(bias_dtype=F16),
                   dict(bias=address(2) + 2), dict(act=4), dict(act=-1), dict(residual=matrix(20, 47, 3)), dict(residual=matrix(19, 48, 3)),
                   dict(y=matrix(20, 49, 4)), dict(z=matrix(21, 48, 5)), dict(y=matrix(20, 48, 3, stride=64)), dict(y=matrix(20, 48)),
                   dict(y=matrix(20, 48, 1)), dict(y=matrix(20, 48, 5)), dict(z=matrix(20, 48, 3)), dict(z=matrix(20, 48)),
                   dict(y=matrix(20, 48, 2)), dict(x=None), dict(weight=None), dict(y=None)):
        assert call(ctx, **change) == BAD, change
    back = Call(lib.abcd_linear_backward, dy=matrix(20, 48), x=matrix(20, 64, 1), weight=matrix(48, 64, 2), act=ab.ABCD_SILU,
                z=matrix(20, 48, 3), dx=matrix(20, 64, 4), dweight=matrix(48, 64, 5), dbias=address(6), bias_dtype=BF16)
    assert back(ctx) == WORKSPACE
    assert back(ctx, act=ab.ABCD_NO_ACTIVATION, z=None) == WORKSPACE
    for change in (dict(z=None), dict(dy=matrix(20, 47)), dict(dx=matrix(20, 63, 4)), dict(dweight=matrix(48, 64, 5, F32)),
                   dict(dx=matrix(20, 64, 1)), dict(dx=matrix(20, 64)), dict(dweight=matrix(48, 64, 2)), dict(dx=matrix(20, 64, 5)),
                   dict(dbias=address(4)), dict(bias_dtype=F16), dict(dbias=address(6) + 1), dict(act=9), dict(dy=None), dict(x=None)):
        assert back(ctx, **change) == BAD, change


def norm(kind=ab.ABCD_LAYER_NORM, weight=address(20), bias=address(21), eps=1e-5, mean=address(22), rstd=address(23)):
    return ab.abcd_norm(kind, weight, bias, eps, mean, rstd)


def test_residual_norm_refusals(lib, ctx):
    x, f, y, n = (matrix(8, 64, k) for k in range(4))
    call = Call(lib.abcd_residual_norm, x=x, f=f, after=norm(), before=norm(), gate=address(24), kind=BF16, scale=1.0, y=y, n=n)
    rms = ab.ABCD_RMS_NORM
    for change in (dict(f=matrix(8, 63, 1)), dict(y=matrix(7, 64, 2)), dict(n=None), dict(before=None), dict(kind=F16), dict(gate=address(24) + 1),
                   dict(after=norm(kind=2)), dict(after=norm(eps=-1.0)), dict(after=norm(eps=float("nan"))), dict(before=norm(weight=address(20) + 1)),
                   dict(before=norm(mean=None)), dict(after=norm(rstd=None)), dict(after=norm(kind=rms)), dict(scale=float("inf")),
                   dict(n=y), dict(n=matrix(8, 64, 0, stride=72)), dict(y=matrix(8, 64, 1.0 / 8192)), dict(after=norm(mean=address(22) + 2)),
                   dict(x=None), dict(y=None), dict(f=matrix(8, 64, 1, F32))):
        assert call(ctx, **change) == BAD, change
    back = Call(lib.abcd_residual_norm_backward, dy=matrix(8, 64, 4), dn=matrix(8, 64, 5), x=x, f=f, after=norm(), before=norm(), gate=address(24),
                kind=F32, scale=1.0, dx=matrix(8, 64, 6), df=matrix(8, 64, 7), dgate=address(25), aw=address(26), ab=address(27), bw=address(28), bb=address(29))
    assert back(ctx) == WORKSPACE
    assert back(ctx, dy=None) == WORKSPACE
    assert back(ctx, dx=matrix(8, 64, 4), df=matrix(8, 64, 5)) == WORKSPACE       # over dy and dn
    assert back(ctx, before=None, dn=None, bw=None, bb=None) == WORKSPACE
    for change in (dict(dn=None), dict(before=None), dict(dy=None, dn=None, before=None, bw=None, bb=None), dict(after=norm(mean=None, rstd=None)),
                   dict(after=None), dict(before=None, dn=None), dict(df=matrix(8, 64, 6)), dict(dx=matrix(8, 64, 4, stride=80)),
                   dict(dgate=address(25) + 2), dict(kind=F16), dict(dx=matrix(8, 63, 6)), dict(scale=float("nan")), dict(x=None)):
        assert back(ctx, **change) == BAD, change
    one = matrix(8, 64, 0.5)
    assert lib.abcd_residual_norm(None, ref(x), ref(f), None, None, None, BF16, 1.0, ref(one), None) == BAD


def test_residual_norm_refuses_vectors_that_overlap(lib, ctx):
    """What a call writes of vectors lies apart from all else that it is given, and its matrices from the vectors."""
    x, f, y, n = (matrix(8, 64, k) for k in range(4))
    first = dict(weight=address(20), bias=address(21), mean=address(22), rstd=address(23))
    second = dict(weight=address(24), bias=address(25), mean=address(26), rstd=address(27))
    call = Call(lib.abcd_residual_norm, x=x, f=f, after=norm(**first), before=norm(**second), gate=address(28), kind=BF16, scale=1.0, y=y, n=n)
    assert call(ctx) == ab.ABCD_ERR_CUDA              # all that is missing: a GPU
    shared = dict(after=norm(**{**first, "weight": address(28)}), before=norm(**{**second, "weight": address(28), "bias": address(21)}))
    assert call(ctx, **shared) == ab.ABCD_ERR_CUDA    # what is only read
    close_by = address(22) + 8 * 4
    assert call(ctx, after=norm(**{**first, "rstd": close_by})) == ab.ABCD_ERR_CUDA
    for change in (dict(after=norm(**{**first, "rstd": close_by - 4})), dict(after=norm(**{**first, "mean": address(20) + 64 * 2 - 4})),
                   dict(before=norm(**{**second, "mean": address(22)})), dict(before=norm(**{**second, "rstd": address(0) + 8 * 64 * 2 - 4})),
                   dict(before=norm(**{**second, "mean": address(1)})), dict(before=norm(**{**second, "rstd": address(2)})),
                   dict(after=norm(**{**first, "mean": address(28)})), dict(y=matrix(8, 64, 24)), dict(n=matrix(8, 64, 28)), dict(n=matrix(8, 64, 21))):
        assert call(ctx, **change) == BAD, change
    # between a matrix's rows
    wide = dict(x=matrix(8, 64, 0, stride=256), y=matrix(8, 64, 2, stride=256))
    assert call(ctx, **wide, gate=address(2) + 64 * 2) == ab.ABCD_ERR_CUDA
    assert call(ctx, **wide, gate=address(2) + 64 * 2 - 2) == BAD
    back = Call(lib.abcd_residual_norm_backward, dy=matrix(8, 64, 4), dn=matrix(8, 64, 5), x=x, f=f, after=norm(**first), before=norm(**second),
                gate=address(28), kind=F32, scale=1.0, dx=matrix(8, 64, 6), df=matrix(8, 64, 7), dgate=address(30), aw=address(31), ab=address(32),
                bw=address(33), bb=address(34))
    assert back(ctx) == WORKSPACE
    assert back(ctx, **shared) == WORKSPACE
    assert back(ctx, dgate=address(30) + 64 * 4, aw=address(30)) == WORKSPACE
    for change in (dict(dgate=address(28)), dict(aw=address(30) + 64 * 4 - 4), dict(ab=address(33)), dict(bw=address(23)), dict(bb=address(0)),
                   dict(bb=address(4) + 8 * 64 * 2 - 4), dict(aw=address(6)), dict(dgate=address(7)), dict(dx=matrix(8, 64, 22)),
                   dict(df=matrix(8, 64, 24)), dict(bw=address(5)), dict(dx=matrix(8, 64, 28))):
        assert back(ctx, **change) == BAD, change


def packed(rows, cols, at, stride=None, powers=None, power_stride=None):
    groups = -(-cols // 32)
    return ab.abcd_packed8(address(at), address(at + 0.5) if powers is None else powers, rows, cols, stride or 32 * groups, power_stride or groups)


def test_packed_refusals(lib, ctx):
    for name, first in (("abcd_pack8", True), ("abcd_unpack8", False)):
        f = getattr(lib, name)
        call = lambda m, q: f(ctx, *((ref(m), ref(q)) if first else (ref(q), ref(m))))
        m, q = matrix(8, 70), packed(8, 70, 2)
        for a, b in ((matrix(8, 69), q), (matrix(7, 70), q), (None, q), (m, None), (m, packed(8, 70, 2, stride=80)), (m, packed(8, 70, 2, stride=64)),
                     (m, packed(8, 70, 2.0 + 16 / (1 << 20))), (m, packed(8, 70, 2, power_stride=2)), (matrix(8, 70, 2), q), (matrix(8, 70, 2.5), q),
                     (m, packed(8, 70, 0))):
            assert call(a, b) == BAD, (name, a, b)
        assert call(matrix(0, 70), packed(0, 70, 2)) == OK
    call = Call(lib.abcd_gated_ff_backward_packed8, dy=matrix(20, 64), x=packed(20, 64, 1), wg=matrix(96, 64, 2), wu=matrix(96, 64, 3), wd=matrix(64, 96, 4),
                act=ab.ABCD_SILU, gate=packed(20, 96, 5), up=packed(20, 96, 6), dx=matrix(20, 64, 7), dg=matrix(96, 64, 8), du=matrix(96, 64, 9), dd=matrix(64, 96, 10))
    assert call(ctx) == WORKSPACE
    for change in (dict(x=packed(20, 63, 1)), dict(gate=packed(19, 96, 5)), dict(up=None), dict(x=None), dict(act=3), dict(dx=matrix(20, 64, 1)),
                   dict(dd=matrix(64, 96, 5.5)), dict(dg=matrix(96, 64, 6)), dict(dy=None), dict(wd=matrix(64, 95, 4))):
        assert call(ctx, **change) == BAD, change


def test_powers_in_the_codes_are_refused(lib, ctx):
    """Those between the rows of codes are not."""
    at, m = address(2), matrix(8, 70)
    for name in ("abcd_pack8", "abcd_unpack8"):
        def call(powers, apart):
            q = packed(8, 70, 2, stride=256, powers=powers, power_stride=apart)
            return getattr(lib, name)(ctx, *((ref(m), ref(q)) if name == "abcd_pack8" else (ref(q), ref(m))))
        for powers, apart in ((at, 3), (at + 69, 3), (at - 8 * 3 + 1, 3), (at + 7 * 256 + 60, 3), (at + 69, 256), (at + 256 - 2, 256), (at + 62, 512)):
            assert call(powers, apart) == BAD, (name, powers - at, apart)
        for powers, apart in ((at + 70, 256), (at + 253, 256), (at - 8 * 3, 3), (at + 7 * 256 + 70, 3)):
            assert call(powers, apart) == ab.ABCD_ERR_CUDA      # all that is missing: a GPU


def test_matrices_in_8_bits_of_host_memory_are_refused(monkeypatch):
    """Before the library sees an address, as the other tensors are."""
    torch = pytest.importorskip("torch")
    from paper_2608_27735_gb300 import network
    class Context:
        h = None
    def never(*args):
        raise AssertionError("the library was called")
    monkeypatch.setattr(network, "_call", lambda name: never)
    monkeypatch.setattr(network, "_matrix", lambda t, what: (b"", 4, 40))
    q = ab.Packed8(4, 40, "cpu")
    for call in (lambda q: network.abcd_pack8(Context, None, q), lambda q: network.abcd_unpack8(Context, q, None),
                 lambda q: network.abcd_gated_ff_backward_packed8(Context, None, q, None, None, None, "silu", q, q)):
        for bad in (q, None, torch.zeros(4, 40)):
            with pytest.raises(ValueError):
                call(bad)


def test_shared_memory_limits_have_a_place():
    """As the sources' own count in tests/test_network_host.py, with the kernels of the token operators."""
    csrc = os.path.join(os.path.dirname(ab.__file__), "csrc")
    read = lambda name: open(os.path.join(csrc, name)).read()
    table = int(re.search(r"kSmemKernels = (\d+)", read("abcd_internal.cuh"))[1])
    epilogues = re.search(r"enum \{ (kPlain[^}]*) \}", read("ffproduct.cuh"))[1].count(",") + 1
    shapes = len(re.findall(r"return launch_product<\d, \d+, EPI, F32>", read("ffproduct.cuh")))
    rows = len(re.findall(r"return f\(CloseRow<", read("residualnorm.cu")))
    assert epilogues == 5 and shapes == 3 and rows == 14
    # four epilogues in every shape, one in one; three sizes of the sort's tiles
    assert 62 + 10 + 4 * shapes * 2 + 1 + rows * 3 * 2 + 3 <= table
