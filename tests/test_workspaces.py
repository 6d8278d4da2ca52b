"""Where the binding takes the 8-bit product's workspace from: on which stream, in
which capture, how much of it stays, and which tensors a caller may give.

The rules are tested without a GPU on a recording stand-in for torch's allocator and
for the library; what they are for, memory that other work still uses, on the GPU."""
import contextlib
import types
import weakref

import pytest
import torch

from paper_2412_00119_gb300 import bmlp as B

DEV = "cuda:0"
gpu = pytest.mark.gpu
SIZE = 4096


class Tensor:
    """What the binding asks of a tensor on the device."""

    def __init__(self, shape, dtype, device=0, ptr=4096):
        self.shape, self.dtype, self.ptr = torch.Size(shape), dtype, ptr
        self.device = torch.device("cuda", device)
        self.is_cuda = True

    def stride(self, dim=None):
        s = [1] * len(self.shape)
        for i in range(len(s) - 2, -1, -1):
            s[i] = s[i + 1] * self.shape[i + 1]
        return tuple(s) if dim is None else s[dim]

    def data_ptr(self):
        return self.ptr

    def get_device(self):
        return self.device.index

    def element_size(self):
        return self.dtype.itemsize

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def record_stream(self, stream):
        pass


class Device:
    """torch's streams and allocator, and the library, as far as the binding sees them."""

    def __init__(self):
        self.current, self.capturing, self.device = 100, set(), 0
        self.allocated = []          # (stream, bytes) of every block
        self.calls = []              # (stream, workspace, bytes) of every product
        self.room = 1 << 40
        self.size = SIZE             # that the library asks for
        self.live = weakref.WeakSet()
        self.pools = {}              # block -> id of the pool it lies in

    def empty(self, size, dtype, device):
        if size > self.room:
            raise torch.cuda.OutOfMemoryError("no room")
        self.allocated.append((self.current, size))
        t = Tensor((size,), dtype, torch.device(device).index or 0, ptr=1 << 20 | len(self.allocated) << 8)
        self.live.add(t)
        self.pools[t.ptr] = (0, 1) if self.current in self.capturing and self.graph else (0, 0)
        return t

    graph = True                     # captures are torch's own
    backend = "native"

    @contextlib.contextmanager
    def stream(self, s):
        before, self.current = self.current, s.cuda_stream
        yield
        self.current = before

    def snapshot(self):
        return [dict(address=p, total_size=256, segment_pool_id=i) for p, i in self.pools.items()]

    def product(self, *args):
        # (workspace, bytes, stream: the last three)
        self.calls.append((args[-1], args[-3], args[-2]))
        return 0


@pytest.fixture
def dev(monkeypatch):
    d = Device()
    B.bmlp_release_workspaces()
    B._use_torch()
    stream = lambda raw=0, device=None: types.SimpleNamespace(cuda_stream=raw)   # noqa: E731
    cuda = types.SimpleNamespace(
        stream=d.stream, Stream=torch.cuda.Stream, ExternalStream=stream, default_stream=lambda device=None: stream(0),
        current_stream=lambda device=None: stream(d.current), is_current_stream_capturing=lambda: d.current in d.capturing,
        OutOfMemoryError=torch.cuda.OutOfMemoryError, memory_snapshot=d.snapshot, get_allocator_backend=lambda: d.backend)
    fake = types.SimpleNamespace(cuda=cuda, empty=d.empty, **{t: getattr(torch, t) for t in
                                 ("int8", "uint8", "int32", "int64", "float32", "float16", "bfloat16")})
    library = types.SimpleNamespace(bmlp_int8_workspace=lambda n, K, N: d.size, bmlp_int8_matmul=d.product,
                                    bmlp_debug_int8_matmul=d.product, bmlp_int8_sign=d.product,
                                    bmlp_debug_int8_sign=d.product)
    monkeypatch.setattr(B, "_torch", fake)
    monkeypatch.setattr(B, "_raw_stream", lambda device: d.current)
    monkeypatch.setattr(B, "_get_device", lambda: d.device)
    monkeypatch.setattr(B, "_devices", 2)
    monkeypatch.setattr(B, "_lib", library)
    yield d
    B.bmlp_release_workspaces()


def product(n=64, K=128, N=256, device=0, out_device=0, **kw):
    a, w = Tensor((n, K), torch.int8, device), Tensor((N, K), torch.int8, device)
    B.bmlp_int8_matmul(a, w, Tensor((n, N), torch.float32, out_device), **kw)


def signs(n=64, K=128, N=256, **kw):
    a, w = Tensor((n, K), torch.int8), Tensor((N, K), torch.int8)
    B.bmlp_int8_sign(a, w, Tensor((n, (N + 63) // 64), torch.int64), **kw)


@pytest.mark.parametrize("call", [product, signs])
def test_workspace_belongs_to_the_calls_stream(dev, call):
    """torch hands a block that was freed on a stream out again at once, in the order of that
    stream alone: the block has to be one of the stream that the kernels run on."""
    for stream in (None, 100, 42, types.SimpleNamespace(cuda_stream=43), 0):
        del dev.allocated[:], dev.calls[:]
        B.bmlp_release_workspaces()
        call(stream=stream)
        (on, workspace, size), = dev.calls
        assert size == SIZE and workspace
        assert dev.allocated == [(on, SIZE)], stream
        assert dev.current == 100


def test_workspace_of_any_layout_is_refused():
    """An expanded or strided tensor has fewer bytes of its own from its pointer on than it has
    elements: the kernels would write past them."""
    a, w = torch.zeros((64, 128), dtype=torch.int8), torch.zeros((256, 128), dtype=torch.int8)
    out, words = torch.zeros((64, 256)), torch.zeros((64, 4), dtype=torch.int64)
    for ws in (torch.zeros((1,), dtype=torch.uint8).expand(1 << 24), torch.zeros((4096,), dtype=torch.uint8)[::2],
               torch.zeros((64, 64), dtype=torch.uint8)[:, :32], torch.zeros((8, 4), dtype=torch.float32).t()):
        with pytest.raises(ValueError, match="workspace"):
            B.bmlp_int8_matmul(a, w, out, workspace=ws)
        with pytest.raises(ValueError, match="workspace"):
            B.bmlp_int8_sign(a, w, words, workspace=ws)


def test_tensors_of_another_device_are_refused(dev):
    """The kernels run on the current device, where another one's memory would be a fault."""
    i8, f32 = torch.int8, torch.float32
    reached = []
    B._lib.bmlp_quantize_rows = B._lib.bmlp_norm_quantize = lambda *a: reached.append(a) or 0

    def quantize(*where):
        x, q, s = (Tensor(*t, d) for t, d in zip([((4, 8), f32), ((4, 8), i8), ((4,), f32)], where))
        B.bmlp_quantize_rows(x, q, s)

    def norm(*where):
        x, g, q, s, r, t = (Tensor(*t, d) for t, d in zip(
            [((4, 8), f32), ((8,), f32), ((4, 8), i8), ((4,), f32), ((4, 8), f32), ((4, 8), f32)], where))
        B.bmlp_norm_quantize(x, g, q, s, res=r, sum_out=t)

    def matmul(*where):
        a, w, o, sa, sw, b, ws = (Tensor(*t, d) for t, d in zip(
            [((64, 8), i8), ((4, 8), i8), ((64, 4), f32), ((64,), f32), ((4,), f32), ((4,), f32), ((64,), torch.uint8)], where))
        B.bmlp_int8_matmul(a, w, o, sa, sw, b, workspace=ws)

    def sign(*where):
        a, w, o, t, ws = (Tensor(*t, d) for t, d in zip(
            [((64, 8), i8), ((4, 8), i8), ((64, 1), torch.int64), ((4,), torch.int32), ((64,), torch.uint8)], where))
        B.bmlp_int8_sign(a, w, o, t, workspace=ws)

    for call, count in ((quantize, 3), (norm, 6), (matmul, 7), (sign, 5)):
        for wrong in range(count):
            with pytest.raises(ValueError, match="device"):
                call(*[int(i == wrong) for i in range(count)])
        with pytest.raises(ValueError, match="device"):
            call(*[1] * count)
        assert not reached and not dev.calls
        dev.device = 1
        call(*[1] * count)
        dev.device = 0
        call(*[0] * count)
        assert len(reached) + len(dev.calls) == 2
        del reached[:], dev.calls[:]


def test_workspace_in_captures(dev):
    """The address of a captured call's workspace stays in the graph: it has to be a block that
    torch keeps for the graph, or none."""
    def run(stream, capturing, graph, want):
        del dev.allocated[:], dev.calls[:]
        dev.capturing, dev.graph = capturing, graph
        product(stream=stream)
        (on, workspace, size), = dev.calls
        assert on == (100 if stream is None else stream)
        if want:
            assert dev.allocated == [(on, SIZE)] and size == SIZE and dev.pools[workspace] == (0, 1)
        else:
            assert not workspace and size == 0
            # no allocation in a capture that torch knows nothing of, where it may not be allowed
            assert not dev.allocated or 100 in capturing
        given = Tensor((SIZE,), torch.uint8, ptr=1 << 40)
        product(stream=stream, workspace=given)
        assert dev.calls[1] == (on, 1 << 40, SIZE)

    for stream in (None, 100, 42):
        run(stream, {100, 42}, True, True)      # torch's capture, and a stream forked from it
        run(stream, {100, 42}, False, False)    # another runtime's capture
    run(42, {42}, False, False)                 # of a stream that is not the current one
    dev.backend = "cudaMallocAsync"             # whose blocks are no device memory in a capture
    for stream in (None, 42):
        run(stream, {100, 42}, True, False)


def test_workspaces_kept_for_few_streams(dev):
    """What stays with the thread is bounded, however many streams it uses; the last used stay."""
    for stream in range(200, 230):
        dev.current = stream
        for _ in range(3):
            product()
        assert len(dev.live) <= 4
    assert len(dev.allocated) == 30
    for stream in (226, 227, 228, 229, 226, 227):
        dev.current = stream
        product()
    assert len(dev.allocated) == 30
    dev.current = 230                # takes the place of the one unused the longest
    product()
    dev.current = 226
    product()
    assert len(dev.allocated) == 31
    dev.current = 228
    product()
    assert len(dev.allocated) == 32 and len(dev.live) == 4
    dev.size = 2 * SIZE              # a larger one takes a smaller one's place
    product()
    product()
    assert len(dev.allocated) == 33 and len(dev.live) == 4
    B.bmlp_release_workspaces()
    assert len(dev.live) == 0


def test_without_room_for_a_workspace(dev):
    """The product has kernels that need none; a later call may find room again."""
    dev.room = SIZE - 1
    for call in (product, signs):
        for stream in (None, 42):
            del dev.calls[:]
            dev.room = SIZE - 1
            call(stream=stream)
            call(stream=stream)
            assert [c[1:] for c in dev.calls] == [(None, 0)] * 2
            dev.room = SIZE
            call(stream=stream)
            assert dev.calls[2][1] and dev.calls[2][2] == SIZE
        B.bmlp_release_workspaces()


@gpu
def test_product_without_room_on_the_device():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(DEV)
    n, K, N = 1500, 4096, 4096
    g = torch.Generator().manual_seed(1)
    a, w = (torch.randint(-128, 128, s, generator=g).to(torch.int8).to(DEV) for s in ((n, K), (N, K)))
    S = (a.double() @ w.double().t()).to(torch.int32)
    out = torch.full((n, N), -3, dtype=torch.int32, device=DEV)
    B.bmlp_release_workspaces()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    size = B.bmlp_int8_workspace(n, K, N)
    assert size > 40 << 20          # (more than is left over in a segment of torch's)
    total = torch.cuda.get_device_properties(DEV).total_memory
    try:
        # a limit of torch's own allocator
        torch.cuda.set_per_process_memory_fraction((torch.cuda.memory_reserved() + (1 << 20)) / total)
        with pytest.raises(torch.cuda.OutOfMemoryError):
            torch.empty((size,), dtype=torch.uint8, device=DEV)
        B.bmlp_int8_matmul(a, w, out)
        B.bmlp_int8_matmul(a, w, out, stream=torch.cuda.Stream())
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    torch.cuda.synchronize()
    assert torch.equal(out, S)


@gpu
@pytest.mark.parametrize("n,K,N", [(300, 2304, 4000), (100, 4096, 8192), (4000, 1500, 100)])
def test_captures_by_the_driver(n, K, N):
    """Captures that torch does not make, of the current stream and of another: the graph uses no
    memory that torch gives to others."""
    import ctypes as C
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(DEV)
    cu = C.CDLL("libcuda.so.1")

    def ok(rc):
        assert rc == 0, rc
    g = torch.Generator().manual_seed(1)
    a, w = (torch.randint(-128, 128, s, generator=g).to(torch.int8).to(DEV) for s in ((n, K), (N, K)))
    S = (a.double() @ w.double().t()).to(torch.int32)
    size = B.bmlp_int8_workspace(n, K, N)
    out = torch.empty((n, N), dtype=torch.int32, device=DEV)
    given = torch.empty((size,), dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    B.bmlp_int8_matmul(a, w, out)
    for how in ("another", "current", "given"):
        with torch.cuda.stream(s):
            blocks = [torch.empty((size,), dtype=torch.uint8, device=DEV) for _ in range(2)]
            del blocks              # (of which torch may take one in the capture)
        torch.cuda.synchronize()
        raw, graph, exe = C.c_void_p(s.cuda_stream), C.c_void_p(), C.c_void_p()
        ok(cu.cuStreamBeginCapture_v2(raw, 1))
        try:
            if how == "another":
                B.bmlp_int8_matmul(a, w, out, stream=s)
            elif how == "given":
                B.bmlp_int8_matmul(a, w, out, stream=s, workspace=given)
            else:
                with torch.cuda.stream(s):
                    B.bmlp_int8_matmul(a, w, out)
        finally:
            ok(cu.cuStreamEndCapture(raw, C.byref(graph)))
        ok(cu.cuGraphInstantiateWithFlags(C.byref(exe), graph, C.c_ulonglong(0)))
        with torch.cuda.stream(s):
            others = [torch.full((size,), 0x7F, dtype=torch.uint8, device=DEV) for _ in range(3)]
            out.fill_(-3)
            ok(cu.cuGraphLaunch(exe, raw))
        torch.cuda.synchronize()
        assert torch.equal(out, S), how
        assert all((t == 0x7F).all() for t in others), how
        ok(cu.cuGraphExecDestroy(exe))
        ok(cu.cuGraphDestroy(graph))


@gpu
def test_workspace_in_a_forked_capture():
    """torch's capture with a second stream: the block is the graph's, and that stream's."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(DEV)
    n, K, N = 300, 2304, 4000
    g = torch.Generator().manual_seed(1)
    a, w = (torch.randint(-128, 128, s, generator=g).to(torch.int8).to(DEV) for s in ((n, K), (N, K)))
    S = (a.double() @ w.double().t()).to(torch.int32)
    outs = [torch.empty((n, N), dtype=torch.int32, device=DEV) for _ in range(3)]
    s = torch.cuda.Stream()
    B.bmlp_int8_matmul(a, w, outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        current = torch.cuda.current_stream()
        s.wait_stream(current)
        B.bmlp_int8_matmul(a, w, outs[0])
        B.bmlp_int8_matmul(a, w, outs[1], stream=s)
        B.bmlp_int8_matmul(a, w, outs[2], stream=s)
        current.wait_stream(s)
    junk = [torch.full((B.bmlp_int8_workspace(n, K, N),), 0x7F, dtype=torch.uint8, device=DEV) for _ in range(3)]
    for _ in range(3):
        for o in outs:
            o.fill_(-3)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, S) for o in outs)
        assert all((t == 0x7F).all() for t in junk)


@gpu
def test_workspace_beside_work_on_the_current_stream():
    """A block of the workspace's size that was freed on the current stream while kernels that
    write and read it are still queued there; then a product on another stream."""
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(DEV)
    n, K, N = 300, 2304, 4000
    g = torch.Generator().manual_seed(1)
    a, w = (torch.randint(-128, 128, s, generator=g).to(torch.int8).to(DEV) for s in ((n, K), (N, K)))
    S = (a.double() @ w.double().t()).to(torch.int32)
    size = B.bmlp_int8_workspace(n, K, N)
    assert size > 0
    s = torch.cuda.Stream()
    busy = torch.randn((2048, 2048), device=DEV)
    out = torch.empty((n, N), dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    for _ in range(5):
        for _ in range(20):
            busy = busy @ busy
            busy /= busy.abs().amax()
        block = torch.full((size,), 7, dtype=torch.uint8, device=DEV)
        busy = busy @ busy
        busy /= busy.abs().amax()
        seen = block.clone()
        del block
        out.fill_(-3)
        done = torch.cuda.Event()
        done.record()
        # (the outputs' filling ends before the product begins; the current stream then has more work)
        s.wait_event(done)
        B.bmlp_int8_matmul(a, w, out, stream=s)
        torch.cuda.synchronize()
        assert (seen == 7).all() and torch.equal(out, S)
        # without that wait: the block's writer and reader are pending while the product runs
        for _ in range(20):
            busy = busy @ busy
            busy /= busy.abs().amax()
        block = torch.full((size,), 9, dtype=torch.uint8, device=DEV)
        busy = busy @ busy
        busy /= busy.abs().amax()
        seen = block.clone()
        del block
        B.bmlp_int8_matmul(a, w, out, stream=s)
        torch.cuda.synchronize()
        assert (seen == 9).all() and torch.equal(out, S)
