"""What the calls of the 8-bit projections take and keep: pairs, gradients, status and errors."""
import pytest
import torch

from tests import _fp8 as R

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def ops():
    import paper_2509_24899_b200 as pkg
    yield pkg
    torch.cuda.synchronize()
    assert pkg.fp8_last_status() == 0


def randn(*shape, dtype=BF16, seed=0, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * gain).to(dtype)


# ------------------------------------------------------------------------------------------------ pairs
@pytest.mark.parametrize("M", [3, 300])
def test_pairs_whose_tensors_nothing_else_holds(ops, M):
    """The call holds a pair's tensors until its work is on the stream, also where the pair is an iterator that has let go of them and the output could take their place."""
    a, w = ops.quantize_fp8(randn(M, 512, seed=1)), ops.quantize_fp8(randn(M, 512, seed=2))
    want = ops.matmul_fp8(a, w)
    for made in (lambda p: (t.clone(memory_format=torch.preserve_format) for t in p), lambda p: map(torch.Tensor.view_as, p, p), lambda p: [t.clone() for t in p], iter):
        for _ in range(8):
            assert torch.equal(ops.matmul_fp8(made(a), made(w)), want)


def test_what_is_no_pair_is_refused(ops):
    a = ops.quantize_fp8(randn(2, 512))
    for bad in (a[0], a[1], (a[0],), (*a, a[0]), (t[:, :4] for t in a), {a[0]: a[1]}, (a[0], None)):
        with pytest.raises(ValueError):
            ops.matmul_fp8(bad, a)
    for bad in (None, 3):
        with pytest.raises(TypeError):
            ops.matmul_fp8(bad, a)


# ------------------------------------------------------------------------------------------------ status
def product_of(a, w, out):
    """as_matmul_fp8_t of a w^T into rows."""
    import ctypes as C

    from paper_2509_24899_b200 import binding as b
    matrix = [b.as_fp8_matrix_t(m.data.data_ptr(), m.data.stride(0), m.scales.data_ptr(), m.data.shape[0]) for m in (a, w)]
    return b.as_matmul_fp8_t(C.sizeof(b.as_matmul_fp8_t), a.data.shape[1], a.data.shape[0], w.data.shape[0], *matrix, None,
                             b.as_rows_t(out.data_ptr(), b.AS_DTYPE_BF16, out.shape[1], out.shape[0], 0, 0, out.stride(0)))


@pytest.fixture()
def context():
    from paper_2509_24899_b200 import binding
    ctx = binding.as_fp8_create()
    yield ctx
    torch.cuda.synchronize()
    binding.as_fp8_destroy(ctx)


@pytest.mark.parametrize("M,N,K", [(2, 300, 1000), (200, 1536, 6144), (700, 1000, 512), (5000, 1536, 512)])
def test_a_wait_that_runs_out_is_reported_once_and_the_context_stays_usable(ops, context, M, N, K):
    """The time-out in its safe form: a kernel of its own whose wait nothing feeds, on the context's status word.  Products behind it on the stream, before and after
    the word has been read, are right."""
    from paper_2509_24899_b200 import binding
    a, w = ops.quantize_fp8(randn(M, K, seed=1)), ops.quantize_fp8(randn(N, K, seed=2, gain=0.05), block_rows=128)
    want = ops.matmul_fp8(a, w)
    out = [torch.full((M, N), 7.0, dtype=BF16, device="cuda") for _ in range(3)]
    st = torch.cuda.current_stream().cuda_stream
    assert binding.as_fp8_last_status(context, st) == 0
    binding.as_matmul_fp8(context, product_of(a, w, out[0]), st)
    assert binding.as_fp8_last_status(context, st) == 0
    binding.as_fp8_debug_expire_wait(context, 2_000_000, st)                   # about a millisecond
    binding.as_matmul_fp8(context, product_of(a, w, out[1]), st)
    assert binding.as_fp8_last_status(context, st) == binding.AS_ERR_DEVICE_TIMEOUT
    assert binding.as_fp8_last_status(context, st) == 0                        # read and cleared
    binding.as_matmul_fp8(context, product_of(a, w, out[2]), st)
    assert binding.as_fp8_last_status(context, st) == 0
    assert all(torch.equal(o, want) for o in out)
    assert ops.fp8_last_status() == 0                                          # another context's word


def test_expire_wait_refuses(ops, context):
    from paper_2509_24899_b200 import binding
    for ctx, limit in ((None, 1000), (context, 0), (context, -1), (context, 100_000_001)):
        with pytest.raises(ops.AsError) as e:
            binding.as_fp8_debug_expire_wait(ctx, limit, 0)
        assert e.value.status == binding.AS_ERR_INVALID_ARG
    assert binding.as_fp8_last_status(context, 0) == 0


def test_status_read_from_two_streams(ops, context):
    """Reads on one stream while waits run out on another: every time-out is reported, by a read under way or by the next one (by both, where the threads of the kernel that
    waits give up one after the other), and none when all of them are over."""
    import threading

    from paper_2509_24899_b200 import binding
    side, reader = torch.cuda.Stream(), torch.cuda.Stream()
    timeouts, stop = [], threading.Event()

    def read():
        while not stop.is_set():
            timeouts.append(binding.as_fp8_last_status(context, reader.cuda_stream) == binding.AS_ERR_DEVICE_TIMEOUT)

    thread = threading.Thread(target=read)
    thread.start()
    raised = 0
    try:
        for _ in range(100):
            before = sum(timeouts)
            binding.as_fp8_debug_expire_wait(context, 2000, side.cuda_stream)
            raised += 1
            side.synchronize()
            seen = binding.as_fp8_last_status(context, side.cuda_stream) == binding.AS_ERR_DEVICE_TIMEOUT
            n = len(timeouts)
            while len(timeouts) < n + 2 and thread.is_alive():
                pass
            assert seen + sum(timeouts) - before >= 1
    finally:
        stop.set()
        thread.join()
    assert raised == 100 and binding.as_fp8_last_status(context, 0) == 0


def test_an_error_of_a_call_stays_with_it(ops):
    """A context that cannot be made (its allocation is refused inside a stream capture) leaves no error behind for the library's next launch.  In a process of its own, as
    the refusal ends the capture as well."""
    import subprocess
    import sys
    text = """
import torch
from paper_2509_24899_b200 import AsError, HybridAttention, binding, workloads as W
op = HybridAttention.from_workload(W.CONFIGS["tiny"])
x = torch.zeros(8, device="cuda")
refused = False
try:
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        x.add_(1)
        try:
            binding.as_fp8_create()
        except AsError:
            refused = True
except RuntimeError:
    pass
binding.as_hybrid_attn_debug_expire_wait(op.handle, 1000, 0)
print("refused" if refused else "made", op.last_status())
"""
    run = subprocess.run([sys.executable, "-c", text], capture_output=True, text=True, timeout=300)
    assert run.stdout.split()[:1] == ["refused"] and "AsError" not in run.stderr, run.stdout + run.stderr[-2000:]
    from paper_2509_24899_b200 import binding
    assert int(run.stdout.split()[1]) == binding.AS_ERR_DEVICE_TIMEOUT


# ------------------------------------------------------------------------------------------------ gradients
def test_tensors_that_require_gradients_are_refused(ops):
    """Each input, and an output that is given; nothing is refused where gradients are off or the tensor is detached."""
    x, r, w, bias = randn(4, 256, seed=1), randn(4, 256, seed=2), randn(256, seed=3), randn(64, seed=4)
    a8, w8 = ops.quantize_fp8(x), ops.quantize_fp8(randn(64, 256, seed=5), block_rows=128)
    calls = [(x, lambda: ops.rms_norm(x, w, residual=r)), (w, lambda: ops.rms_norm(x, w)), (r, lambda: ops.rms_norm(x, w, residual=r, fp8=True)),
             (r, lambda: ops.rms_norm(x, residual=randn(4, 256), residual_out=r)), (r, lambda: ops.rms_norm(x, out=r)),
             (x, lambda: ops.quantize_fp8(x)), (bias, lambda: ops.matmul_fp8(a8, w8, bias=bias))]
    for tensor, call in calls:
        call()
        tensor.requires_grad_()
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()
        with torch.inference_mode():
            call()
        tensor.requires_grad_(False)
        call()


def test_given_outputs_count_as_modified_in_place(ops):
    """A backward pass that needs a tensor which a call has written since says so."""
    x, w8 = randn(4, 256, seed=1), ops.quantize_fp8(randn(256, 256, seed=5), block_rows=128)
    x8 = ops.quantize_fp8(x)
    for call in (lambda t: ops.rms_norm(x, out=t), lambda t: ops.rms_norm(x, residual=t, residual_out=t), lambda t: ops.rms_norm(x, residual=x, residual_out=t, fp8=True),
                 lambda t: ops.matmul_fp8(x8, w8, out=t)):
        saved, p = randn(4, 256, seed=7), torch.ones(4, 256, dtype=BF16, device="cuda", requires_grad=True)
        loss = (p * saved).sum()
        version = saved._version
        call(saved)
        assert saved._version == version + 1
        with pytest.raises(RuntimeError, match="inplace"):
            loss.backward()
    pair = ops.empty_fp8(4, 256)
    for i, call in enumerate((lambda: ops.quantize_fp8(x, out=pair), lambda: ops.rms_norm(x, fp8=True, out=pair))):
        call()
        assert pair.data._version == pair.scales._version == i + 1
    # inputs are not modified, and inference tensors, which keep no count, are taken
    version = [t._version for t in (x, *x8, *w8)]
    ops.matmul_fp8(x8, w8)
    ops.rms_norm(x, residual=x)
    assert version == [t._version for t in (x, *x8, *w8)]
    with torch.inference_mode():
        out = torch.empty(4, 256, dtype=BF16, device="cuda")
        assert torch.equal(ops.rms_norm(x, out=out), ops.rms_norm(x))
    assert torch.equal(ops.rms_norm(x, out=out), ops.rms_norm(x))


def test_layer_of_parameters(ops):
    """Weights that are a module's parameters are taken as the constants that they are for the layer; what it is called on is refused where it requires a gradient."""
    from paper_2509_24899_b200 import HybridAttention, workloads as W
    from paper_2509_24899_b200.fp8_layer import Fp8AttentionLayer
    wl = W.CONFIGS["tiny"]
    D, rows = wl.H * wl.d, wl.B * wl.N
    data = W.generate(wl, wq_gain=2e-3)
    phi = {n: torch.from_numpy(data[n].view("int16")).cuda().view(BF16) for n in ("wq", "wk")}
    plain = {n: randn(D, D, seed=i, gain=D ** -0.5) for i, n in enumerate("qkvo")} | {"bias_q": randn(D, seed=9), "norm": randn(D, seed=10), "norm_k": None}
    hidden, residual = randn(rows, D, seed=30), randn(rows, D, seed=31)
    attention = HybridAttention.from_workload(wl)
    y, total = Fp8AttentionLayer(attention, plain, phi).forward(hidden, residual)
    layer = Fp8AttentionLayer(attention, {n: None if t is None else torch.nn.Parameter(t) for n, t in plain.items()}, phi)
    got = layer.forward(hidden, residual)
    assert torch.equal(got[0], y) and torch.equal(got[1], total)
    with pytest.raises(ValueError, match="gradient"):
        layer.forward(hidden.requires_grad_(), residual)


# ------------------------------------------------------------------------------------------------ threads
def test_a_context_that_cannot_be_made_holds_no_other_thread_up(ops):
    """Two threads whose calls are the first on a device, where setting its context up is refused (inside a stream capture): each gets its exception, also while the
    other's is being made, which runs Python code.  In a process of its own, as the refusal ends the capture as well."""
    import subprocess
    import sys
    text = """
import threading, time, torch
from paper_2509_24899_b200 import block_fp8
seen = []
class Slow(RuntimeError):
    def __init__(self, status, where):
        seen.append(status)
        time.sleep(1)
block_fp8._calls.set_classes(block_fp8.BlockFp8, Slow)
x = torch.zeros(8, device="cuda")
def call():
    try:
        block_fp8.fp8_last_status()
    except Slow:
        seen.append("raised")
threads = [threading.Thread(target=call) for _ in range(3)]
try:
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        x.add_(1)
        for t in threads:
            t.start()
        for t in threads:
            t.join()
except RuntimeError:
    pass
print(seen.count("raised"), len(seen), max(s for s in seen if s != "raised") > 0)
"""
    run = subprocess.run([sys.executable, "-c", text], capture_output=True, text=True, timeout=120)
    assert run.stdout.split() == ["3", "6", "True"], run.stdout + run.stderr[-2000:]


# ------------------------------------------------------------------------------------------------ C entries
def test_the_product_refuses(ops, context):
    """Arguments that the C entry does not take, one at a time, through the binding; the output stays as it was, and the call without the change runs."""
    from paper_2509_24899_b200 import binding as b
    M, N, K = 20, 48, 200
    a, w = ops.quantize_fp8(randn(M, K, seed=1)), ops.quantize_fp8(randn(N, K, seed=2), block_rows=128)
    out = torch.full((M, N), 7.0, dtype=BF16, device="cuda")

    def rows(data=out.data_ptr(), dtype=b.AS_DTYPE_BF16, head_dim=N, tokens=M, sb=0, sh=0, st=N):
        return b.as_rows_t(data, dtype, head_dim, tokens, sb, sh, st)

    def matrix(m, data=None, pitch=None, scales=None, scale_rows=None):
        first = lambda x, y: y if x is None else x           # noqa: E731
        return b.as_fp8_matrix_t(first(data, m.data.data_ptr()), first(pitch, m.data.stride(0)), first(scales, m.scales.data_ptr()), first(scale_rows, m.data.shape[0]))

    bad = [dict(struct_size=8), dict(cols=0), dict(cols=(1 << 20) + 1), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(out_cols=0), dict(out_cols=(1 << 24) + 1), dict(bias=1),
           dict(a=matrix(a, data=0)), dict(a=matrix(a, data=a.data.data_ptr() + 8)), dict(a=matrix(a, pitch=192)), dict(a=matrix(a, pitch=216)), dict(a=matrix(a, scales=0)),
           dict(a=matrix(a, scales=a.scales.data_ptr() + 2)), dict(a=matrix(a, scale_rows=M - 1)), dict(w=matrix(w, scale_rows=N - 1)), dict(w=matrix(w, data=0)),
           dict(out=rows(data=0)), dict(out=rows(data=out.data_ptr() + 1)), dict(out=rows(dtype=b.AS_DTYPE_F32)), dict(out=rows(head_dim=0)), dict(out=rows(head_dim=20)),
           dict(out=rows(tokens=0)), dict(out=rows(tokens=3)), dict(out=rows(st=-N)), dict(out=rows(st=N - 1)), dict(out=rows(st=0)), dict(out=rows(head_dim=16, sh=8)),
           dict(out=rows(tokens=10, sb=N, st=N))]
    for change in bad:
        args = product_of(a, w, out)
        for field, value in change.items():
            setattr(args, field, value)
        with pytest.raises(ops.AsError) as e:
            b.as_matmul_fp8(context, args, 0)
        assert e.value.status == b.AS_ERR_INVALID_ARG, change
    # more columns in heads that lie apart than an index takes
    args = product_of(a, w, out)
    args.out_cols, args.out, args.w = 1 << 24, rows(head_dim=1 << 23, sh=1 << 30, st=1 << 40), matrix(w, scale_rows=1 << 24)
    with pytest.raises(ops.AsError) as e:
        b.as_matmul_fp8(context, args, 0)
    assert e.value.status == b.AS_ERR_UNSUPPORTED
    torch.cuda.synchronize()
    assert bool((out == 7).all())
    args = product_of(a, w, out)
    args.rows, args.a, args.out = 0, matrix(a, scale_rows=0), rows(tokens=0)
    b.as_matmul_fp8(context, args, 0)                                          # no rows: nothing to do
    torch.cuda.synchronize()
    assert bool((out == 7).all())
    b.as_matmul_fp8(context, product_of(a, w, out), 0)
    R.check_matmul(out, a, w)


def test_norm_and_8_bit_form_through_the_binding(ops):
    import ctypes as C

    from paper_2509_24899_b200 import binding as b
    x, y = randn(5, 200, seed=1), torch.empty(5, 200, dtype=BF16, device="cuda")
    form = ops.empty_fp8(5, 200)
    rows = [b.as_rows_t(t.data_ptr(), b.AS_DTYPE_BF16, 200, 5, 0, 0, 200) for t in (x, y)]
    matrix = b.as_fp8_matrix_t(form.data.data_ptr(), form.data.stride(0), form.scales.data_ptr(), 5)
    args = b.as_rms_norm_t(struct_size=C.sizeof(b.as_rms_norm_t), cols=200, rows=5, x=rows[0], out=rows[1], eps=1e-6)
    b.as_rms_norm(args, 0)
    assert torch.equal(y, ops.rms_norm(x))
    b.as_quantize_fp8(b.as_quantize_fp8_t(C.sizeof(b.as_quantize_fp8_t), 200, 5, rows[0], matrix, 1, 0), 0)
    assert all(torch.equal(s.view(torch.uint8), t.view(torch.uint8)) for s, t in zip(form, ops.quantize_fp8(x)))
    args.eps = -1.0
    with pytest.raises(ops.AsError):
        b.as_rms_norm(args, 0)
