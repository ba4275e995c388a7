"""The 8-bit product behind kernels that let it start early: whatever the kernel in front does, the product sees what it wrote."""
import pytest
import torch

import paper_2608_05483_b200 as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# Lets the next kernel of the stream start at once, and writes only a good while later.  (The delay is bounded.)
LATE = r"""
extern "C" __global__ void late_copy(uint4* to, const uint4* from, long long n, long long cycles) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const long long t0 = clock64();
    while (clock64() - t0 < cycles) {}
    for (long long i = blockIdx.x * (long long)blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) to[i] = from[i];
}
"""


class _Late:
    def __init__(self):
        from cuda.bindings import driver, nvrtc
        self.driver = driver
        torch.zeros(1, device=DEV)                      # the primary context is current
        major, minor = torch.cuda.get_device_capability()
        err, prog = nvrtc.nvrtcCreateProgram(LATE.encode(), b"late.cu", 0, [], [])
        assert int(err) == 0
        opts = [f"--gpu-architecture=sm_{major}{minor}".encode()]
        assert int(nvrtc.nvrtcCompileProgram(prog, len(opts), opts)[0]) == 0
        size = nvrtc.nvrtcGetCUBINSize(prog)[1]
        image = b" " * size
        assert int(nvrtc.nvrtcGetCUBIN(prog, image)[0]) == 0
        err, self.module = driver.cuModuleLoadData(image)
        assert int(err) == 0
        err, self.fn = driver.cuModuleGetFunction(self.module, b"late_copy")
        assert int(err) == 0

    def copy(self, to, source, cycles=400_000):
        """to and source: uint8 storage of one size, a multiple of 16 bytes, packed."""
        import ctypes
        assert to.is_contiguous() and source.is_contiguous() and to.numel() == source.numel() and to.numel() % 16 == 0
        assert to.data_ptr() % 16 == 0 and source.data_ptr() % 16 == 0
        values = (to.data_ptr(), source.data_ptr(), to.numel() // 16, cycles)
        types = (ctypes.c_void_p, ctypes.c_void_p, ctypes.c_longlong, ctypes.c_longlong)
        err, = self.driver.cuLaunchKernel(self.fn, 16, 1, 1, 256, 1, 1, 0, torch.cuda.current_stream().cuda_stream, (values, types), 0)
        assert int(err) == 0


@pytest.fixture(scope="module")
def late():
    return _Late()


def _case(m, k, ns, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV)
    f8 = torch.float8_e4m3fn
    x, xs = (rnd(m, k) * 60).clamp(-448, 448).to(f8), torch.exp(rnd(m, -(-k // 128))) * 0.01
    ws = [torch.exp(rnd(-(-n // 128), -(-k // 128))) * 0.01 for n in ns]
    pairs = [[(rnd(n, k) * 60).clamp(-448, 448).to(f8) for n in ns] for _ in range(2)]
    return x, xs, ws, pairs


# one row (clusters that split K), narrow tiles, single CTAs of 128 rows, pairs
@pytest.mark.parametrize("m,k,ns", [(1, 4096, (4096, 1024)), (40, 2048, (1024,)), (128, 1024, (2048,)), (300, 1024, (1000, 512))])
def test_weights_written_by_a_kernel_that_signals_early(late, m, k, ns):
    x, xs, ws, (a, b) = _case(m, k, ns, m)
    want = [P.gemm_fp8(x, xs, w, ws) for w in (a, b)]
    assert not torch.equal(want[0][0], want[1][0])
    live = [w.clone() for w in a]
    raw = lambda t: t.view(torch.uint8).view(-1)
    torch.cuda.synchronize()

    def step(source):
        for t, s in zip(live, source):
            late.copy(raw(t), raw(s))
        return P.gemm_fp8(x, xs, live, ws)

    for source, w in ((b, want[1]), (a, want[0]), (b, want[1])):
        got = step(source)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, w))
    # the same steps in a graph
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        captured = [step(source) for source in (a, b, a)]
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip(captured, (want[0], want[1], want[0])):
            assert all(torch.equal(p, q) for p, q in zip(got, w))


@pytest.mark.parametrize("m,k,ns", [(1, 4096, (4096, 1024)), (40, 2048, (1024,)), (128, 1024, (2048,)), (300, 1024, (1000, 512))])
def test_x_and_scales_written_by_a_kernel_that_signals_early(late, m, k, ns):
    """With weights_ready only the weights may be read early: x and every scale come behind the kernel in front."""
    x, xs, ws, (a, _) = _case(m, k, ns, m + 1)
    want = P.gemm_fp8(x, xs, a, ws)
    pad = lambda t: torch.zeros(-(-t.numel() * t.element_size() // 16) * 16, dtype=torch.uint8, device=DEV)
    bytes_of = lambda t: t.contiguous().view(-1).view(torch.uint8)
    for part in range(3):
        new = [x, xs, ws[0]][part]
        source, store = pad(new), pad(new)
        source[:new.numel() * new.element_size()] = bytes_of(new)
        held = store[:new.numel() * new.element_size()].view(new.dtype).view(new.shape)
        args = [x, xs, a, list(ws)]
        if part < 2:
            args[part] = held
        else:
            args[3][0] = held
        torch.cuda.synchronize()
        late.copy(store, source)
        got = P.gemm_fp8(*args, weights_ready=True)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), part


@pytest.mark.parametrize("m,k,ns", [(1, 4096, (4096, 1024)), (40, 2048, (1024,)), (128, 1000, (2048, 8)), (300, 1024, (1000, 512)), (1111, 656, (520,))])
def test_weights_ready_gives_the_same_bits(m, k, ns):
    x, xs, ws, (a, _) = _case(m, k, ns, m + 2) if k % 16 == 0 else _case(m, k // 16 * 16, ns, m + 2)
    torch.cuda.synchronize()
    for _ in range(5):
        early = P.gemm_fp8(x, xs, a, ws, weights_ready=True)
        behind = P.gemm_fp8(x, xs, a, ws)
        assert all(torch.equal(p, q) for p, q in zip(early, behind))
