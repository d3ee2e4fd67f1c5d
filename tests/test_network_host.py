"""The host's side of the network calls without a GPU: streams of what the package allocates, calls on
a null context, the library's tables."""
import ctypes as C
from types import SimpleNamespace

import pytest

import paper_2608_27735_gb300 as ab


class Stream:
    def __init__(self, name, log):
        self.name, self.log = name, log

    def wait_stream(self, other):
        self.log.append(("wait", self.name, other.name))


class Tensor:
    def __init__(self, log):
        self.log = log

    def data_ptr(self):
        return 0x1000

    def record_stream(self, stream):
        self.log.append(("record", stream.name))


class Library:
    """The library's calls that reserve a workspace, and what they were called after."""

    def __init__(self, log):
        self.log = log

    def abcd_network_workspace_size(self, rows, cols, ff, dtype, out):
        out._obj.value = 1024 * rows
        return ab.ABCD_OK

    def abcd_workspace_size(self, gaussians, pairs, pixels, out):
        out._obj.value = 1024 * gaussians
        return ab.ABCD_OK

    def abcd_set_network_workspace(self, h, p, n):
        self.log.append(("set",))
        return ab.ABCD_OK

    abcd_set_workspace = lambda self, *a: self.abcd_set_network_workspace(*a[:3])


@pytest.fixture
def context(monkeypatch):
    """A context on a stream "own" while the current one is "current", and the log of both."""
    log = []
    current = Stream("current", log)
    torch = SimpleNamespace(uint8=None, empty=lambda *a, **k: Tensor(log),
                            cuda=SimpleNamespace(current_stream=lambda device: current))
    library = Library(log)
    monkeypatch.setattr(ab, "_torch", lambda: torch)
    monkeypatch.setattr(ab, "lib", lambda: library)
    c = ab.Context.__new__(ab.Context)
    c.h, c.device, c.stream, c.workspace, c.limits = None, 0, Stream("own", log), None, (0, 0, 0)
    c.network_workspace, c.network_bytes = None, 0
    return c, current, log


def test_network_workspace_waits_for_the_stream_it_was_allocated_on(context):
    """The allocator hands out memory that kernels of the current stream may still write: the
    context's stream waits for them before it clears the workspace, and the memory for the context's."""
    c, current, log = context
    c.reserve_network(4, 8, 8)
    assert log == [("wait", "own", "current"), ("record", "own"), ("set",)]
    c.reserve_network(2, 8, 8)                          # no more than it has
    assert len(log) == 3
    c.reserve_network(8, 8, 8)
    assert log[3:] == log[:3]


def test_network_workspace_on_the_current_stream_waits_for_nothing(context):
    c, current, log = context
    c.stream = current
    c.reserve_network(4, 8, 8)
    assert log == [("record", "current"), ("set",)]


def test_workspace_waits_for_the_stream_it_was_allocated_on(context):
    """The renderer's workspace likewise; one that is replaced is kept for the calls that use it."""
    c, current, log = context
    c.reserve(4, 8, 8)
    assert log == [("wait", "own", "current"), ("record", "own"), ("set",)]
    c.reserve(4, 8, 8)                                  # no more than it has
    assert len(log) == 3
    c.reserve(8, 8, 8)
    assert log[3:] == log[:3]


def test_block_waits_for_the_stream_its_buffers_were_allocated_on(context, monkeypatch):
    """Every buffer of a FeedForwardBlock is the context's stream's to use, and kept for its calls."""
    from paper_2608_27735_gb300 import network
    c, current, log = context
    made = []

    def allocate(*a, **k):
        t = Tensor(log)
        t.shape, t.dtype, t.device = (a[0] if isinstance(a[0], tuple) else a), None, None
        made.append(t)
        return t

    torch = SimpleNamespace(uint8=None, float32=None, empty=allocate,
                            empty_like=lambda t: allocate(t.shape), cuda=ab._torch().cuda)
    for module in (ab, network):
        monkeypatch.setattr(module, "_torch", lambda: torch)
    held = []
    monkeypatch.setattr(ab.Context, "hold", lambda self, *tensors: held.extend(tensors))
    weights = {"norm_w": (8,), "norm_b": (8,), "w_gate": (16, 8), "w_up": (16, 8), "w_down": (8, 16)}
    w = {k: SimpleNamespace(shape=s, dtype=None, device=None) for k, s in weights.items()}
    network.FeedForwardBlock(c, w, 4)
    assert {id(t) for t in made} == {id(t) for t in held}


def test_clear_status_rejects_a_null_context():
    """In a process of its own, which a read through the null pointer would end."""
    import os
    import subprocess
    import sys
    ab.build()
    code = "import paper_2608_27735_gb300 as ab; print(ab.lib().abcd_clear_status(None))"
    run = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True,
                         cwd=os.path.dirname(os.path.dirname(ab.HEADER)))
    assert (run.returncode, run.stdout.strip()) == (0, str(ab.ABCD_ERR_WORKSPACE))


def test_every_kernel_with_much_shared_memory_has_a_place():
    """A context remembers which kernels it has raised the shared memory limit of; one that finds no place
    would be asked for again in every launch.  Counted from the sources: layer norm's row shapes (three
    types, forward and backward, rows on 16-byte boundaries and not) whose rows ahead take more than
    47 KB, the products' three shapes, three epilogues and two widths, and the renderer's kernels."""
    import os
    import re
    csrc = os.path.join(os.path.dirname(ab.__file__), "csrc")
    read = lambda name: open(os.path.join(csrc, name)).read()
    shapes = re.findall(r"return f\(RowShape<(\d+), V, (\w+), BWD, SHIFT>", read("layernorm.cu"))
    assert len(shapes) == 9
    kernels = set()
    for kind, size in enumerate((4, 2, 2)):
        for backward in (False, True):
            for shift in (False, True):
                for lanes, vectors in shapes:
                    lanes, nv = int(lanes), (16 if backward else 32) * size // 16 if vectors == "N" else int(vectors)
                    ahead = (2 if backward else 1) * (max(lanes, 256) // lanes) * (lanes * nv + shift) * 16
                    ring = (3 if 4 * ahead > 100 * 1024 else 4) * ahead
                    sums = 2 * lanes * nv * 16 // size * 4 if backward else 0
                    if max(ring, sums) > 47 * 1024:
                        kernels.add((kind, backward, shift, lanes, nv))
    products = len(re.findall(r"return launch_product<\d, \d+, EPI, F32>", read("ffproduct.cuh"))) * 3 * 2
    assert products == 18
    renderer = 4 + 2 + 1 + 1 + 2                        # visibility, tile rows, ranges, place, loss
    table = int(re.search(r"kSmemKernels = (\d+)", read("abcd_internal.cuh"))[1])
    assert len(kernels) == 62 and len(kernels) + products + renderer <= table


def test_overlap_of_matrices_is_that_of_their_elements(tmp_path):
    """network.cuh's overlap() against every byte of both matrices: rows apart or not, in one buffer,
    equally far apart or not."""
    import os
    import subprocess
    from paper_2608_27735_gb300 import _build
    src, exe = tmp_path / "overlap.cu", tmp_path / "overlap"
    src.write_text(r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "network.cuh"
using namespace abcd;
static int draw(int n) { return rand() / 7 % n; }
int main() {
  long both[2] = {0, 0}, wrong = 0;
  srand(5);
  for (long k = 0; k < 400000; ++k) {
    abcd_matrix m[2];
    const int common = 1 + draw(12);
    for (auto& q : m) {
      q.dtype = draw(2) ? ABCD_F32 : ABCD_F16;
      const int e = (int)elem_size(q.dtype);
      q.rows = draw(7);
      q.cols = 1 + draw(6);
      q.stride = draw(2) ? q.cols + draw(8) : std::max<long long>(q.cols, common * 4 / e);
      q.data = (void*)(uintptr_t)(4096 + e * draw(40));
    }
    std::vector<char> seen(8192, 0);
    bool meet = false;
    for (int w = 0; w < 2; ++w)
      for (long long r = 0; r < m[w].rows; ++r)
        for (long long b = 0; b < m[w].cols * (long long)elem_size(m[w].dtype); ++b) {
          char& c = seen[(uintptr_t)m[w].data - 4096 + r * m[w].stride * elem_size(m[w].dtype) + b];
          if (w && c) meet = true;
          if (!w) c = 1;
        }
    ++both[meet];
    wrong += overlap(&m[0], &m[1]) != meet || overlap(&m[1], &m[0]) != meet;
  }
  printf("%ld %ld %ld\n", both[0], both[1], wrong);
}
""")
    subprocess.run([_build.nvcc(), *_build.ARCH, *_build.FLAGS, "-I", _build.CSRC, str(src), "-o", str(exe)], check=True)
    apart, meeting, wrong = map(int, subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split())
    assert apart > 50000 and meeting > 50000 and wrong == 0
