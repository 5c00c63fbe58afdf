"""Projections in 8-bit floating point with a scale per block of 128 (pat_op_f8_pack_weight, pat_op_f8_gemm) against a plain implementation in 64 bits."""
import pytest
import torch

from gpu_util import DEV
from operator_refs import check, eight_bit, project

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pat():
    import paper_2605_23945_amd as p
    p.load_library()
    return p


def _x(shape, seed, dtype=torch.float32, std=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


def _run(pat, x, w, **kw):
    return pat.pat_op_f8_gemm(*pat.pat_op_f8_pack_weight(w.to(DEV)), w.shape[0], x.to(DEV), **kw)


def _check(pat, m, n, k, x_dtype=torch.float32, y_dtype=torch.float32, rows=None, seed=0):
    x, w = _x((m, k), seed + m, x_dtype), _x((n, k), seed + n + 1, torch.bfloat16, 0.05)
    got = _run(pat, x, w, y_dtype=y_dtype)
    assert got.dtype == y_dtype and got.shape == (m, n)
    rows = list(range(m)) if rows is None else rows
    ref, allow = project(eight_bit(x[rows], 1), eight_bit(w, 128))
    check(got[rows], ref, allow)


@pytest.mark.parametrize("m", [1, 2, 8, 15, 16, 17, 31, 32, 33, 64, 65, 100, 129, 257])
def test_batches(pat, m):
    _check(pat, m, 272, 384, torch.bfloat16, torch.bfloat16)


@pytest.mark.parametrize("n,k", [(1, 1), (3, 5), (16, 128), (17, 127), (130, 129), (256, 1000), (1000, 77), (64, 4096), (127, 640), (513, 300), (4096, 513)])
@pytest.mark.parametrize("m", [1, 5, 40, 200])
def test_odd_sizes(pat, m, n, k):
    _check(pat, m, n, k)


@pytest.mark.parametrize("x_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("y_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m", [3, 70, 300])
def test_types(pat, m, x_dtype, y_dtype):
    _check(pat, m, 384, 512, x_dtype, y_dtype)


@pytest.mark.parametrize("y_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (8, 12288, 1024), (16, 8208, 2048), (16, 8208, 2176), (5, 3000, 28672), (12, 300, 6912), (40, 24000, 300), (27, 5120, 2048), (64, 2048, 6912),
                                   (251, 4096, 4096), (600, 3000, 1111), (1500, 7168, 1024), (5003, 1024, 1024), (40, 32000, 256), (16, 256, 28672), (300, 200, 11008),
                                   (120, 20000, 300), (1000, 7170, 700), (700, 12304, 520), (300, 11008, 256), (100, 300, 5000), (70, 100, 6912)])
def test_larger_products(pat, m, n, k, y_dtype):
    """Every tile of weights, one to eight of them a workgroup, four and eight waves, K whole and in slices, ends inside tiles."""
    _check(pat, m, n, k, torch.bfloat16, y_dtype, rows=sorted({0, m // 3, m // 2, m - 1}), seed=5)


def test_the_forms_are_bit_exact(pat):
    """The identity on either side lets the other side's 8-bit values through unchanged: a weight's, and an activation's, ties, subnormal
    numbers of the format, blocks that end on a power of two and blocks of zeros among them."""
    k = 300
    t = _x((140, k), 1, torch.bfloat16, 3.0)
    t[0, :128] = torch.linspace(-448, 448, 128).to(torch.bfloat16)
    t[1, :128] = 2.0 ** torch.arange(-64, 64).float()          # from far below the block's smallest step up to its largest
    t[2] = 0
    t[3, 128:256] = 3.5                                        # 448 / 2^7: the border of a scale
    t[4, 128:256] = 3.515625                                   # the bf16 value above it
    t[5, :16] = torch.tensor([17, 19, 21, 23, 25, 27, 29, 31, -17, -19, 34, 38, 42, 46, 1.0625, 1.1875]).to(torch.bfloat16)      # ties
    t[6] *= 2.0 ** -100
    t[7] *= 2.0 ** 100
    eye = torch.eye(k)
    got = _run(pat, eye, t)                                    # y[i, j] = w[j, i]
    assert torch.equal(got.cpu().double().t(), eight_bit(t, 128))
    got = _run(pat, t, eye)
    assert torch.equal(got.cpu().double(), eight_bit(t, 1))
    got = _run(pat, t.float(), eye)
    assert torch.equal(got.cpu().double(), eight_bit(t, 1))


def test_scales_of_all_sizes(pat):
    """Blocks from 2^-126 up to the largest numbers; where the two scales' product leaves fp32's range the products do too."""
    k = 128
    eye = torch.eye(k)
    for e in (-126, -110, -60, 0, 60, 100, 118):
        t = _x((20, k), 3).clamp(-3, 3) * 2.0 ** e
        assert torch.equal(_run(pat, t, eye).cpu().double(), eight_bit(t, 1)), e


@pytest.mark.parametrize("m,n,k", [(1, 130, 200), (40, 130, 200), (140, 130, 200)])
def test_scales_of_all_sizes_in_products(pat, m, n, k):
    """Exponents of x and W that cancel, or leave a large or a small result, and one whose scales' product is no fp32 number."""
    for ex, ew in ((-110, 110), (110, -110), (60, 50), (-60, -50), (-100, 20), (-126, 0), (-70, -70), (0, 118)):
        x, w = (_x((m, k), 5).clamp(-3, 3) * 2.0 ** ex), (_x((n, k), 6).clamp(-3, 3) * 2.0 ** ew)
        got = _run(pat, x, w)
        xq, wq = eight_bit(x, 1), eight_bit(w, 128)
        ref, allow = project(xq, wq)
        check(got, ref, allow + k * 2.0 ** -149)               # and a step of fp32's smallest numbers for each sum
    x, w = torch.full((m, k), 2.0 ** 100), torch.full((n, k), -2.0 ** 90)
    assert bool((_run(pat, x, w) == float("-inf")).all())      # 2^190
    x, w = torch.full((m, k), 2.0 ** -100), torch.full((n, k), 2.0 ** -90)
    assert not bool(_run(pat, x, w).any())                     # 2^-190


def test_what_is_not_finite_becomes_nan_and_leaves_the_scale_alone(pat):
    x = _x((3, 256), 2)
    x[1, 5], x[2, 200] = float("inf"), float("nan")
    w = _x((32, 256), 3)
    got = _run(pat, x, w).cpu()
    ref, allow = project(eight_bit(x[:1], 1), eight_bit(w, 128))
    check(got[:1], ref, allow)
    assert bool(got[1:].isnan().all())
    w[7, 9] = float("-inf")
    got = _run(pat, x[:1], w).cpu()
    assert bool(got[0, 7].isnan()) and int(got.isnan().sum()) == 1
    w[7, 9] = 0
    ref, allow = project(eight_bit(x[:1], 1), eight_bit(w, 128))
    keep = [i for i in range(32) if i != 7]
    check(got[:, keep], ref[:, keep], allow[:, keep])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(4, 100, 130), (90, 333, 256), (300, 1024, 640)])
def test_adding_to_y_and_rows_with_strides(pat, m, n, k, dtype):
    xw, yw = _x((m, k + 8), 7, dtype), _x((m, n + 5), 8, dtype)
    w = _x((n, k + 3), 9)
    x, y = xw.to(DEV)[:, 1:k + 1], yw.to(DEV)
    pw = pat.pat_op_f8_pack_weight(w.to(DEV)[:, 2:k + 2])
    pat.pat_op_f8_gemm(*pw, n, x, y[:, 2:n + 2], mode=1)
    ref, allow = project(eight_bit(xw[:, 1:k + 1], 1), eight_bit(w[:, 2:k + 2], 128))
    y0 = yw[:, 2:n + 2].double()
    check(y[:, 2:n + 2], ref + y0, allow + 2.0 ** -23 * (ref.abs() + y0.abs()))
    assert torch.equal(y[:, :2].cpu(), yw[:, :2]) and torch.equal(y[:, n + 2:].cpu(), yw[:, n + 2:])


def test_single_columns_of_any_stride(pat):
    w, x = _x((40, 1), 1), _x((5, 1), 2)
    w2, x2 = w.t().contiguous().t(), x.t().contiguous().t()    # [n, 1] with strides (1, n)
    assert torch.equal(_run(pat, x2, w2), _run(pat, x, w))
    y = torch.full((1, 5), float("nan"), device=DEV).t()       # and a result of one column
    assert torch.equal(_run(pat, x2, w2[:1], y=y), _run(pat, x, w[:1])) and not bool(y.isnan().any())


def test_no_rows(pat):
    pw = pat.pat_op_f8_pack_weight(_x((32, 64), 1).to(DEV))
    assert pat.pat_op_f8_gemm(*pw, 32, torch.empty(0, 64, device=DEV)).shape == (0, 32)


@pytest.mark.parametrize("m,n,k", [(5, 300, 130), (40, 300, 520), (300, 300, 640), (700, 12304, 520)])
def test_scales_of_the_padding_are_set(pat, m, n, k):
    """A weight's scales go four to a word: what a shorter last word holds beside them is defined, whatever was in the memory before."""
    lib = pat.load_library()
    w, x = _x((n, k), 1, torch.bfloat16, 0.05).to(DEV), _x((m, k), 2, torch.bfloat16).to(DEV)
    packed, scales = pat.pat_op_f8_pack_weight(w)
    again = torch.full_like(scales, 255)
    assert lib.pat_op_f8_pack_weight(w.data_ptr(), 1, k, n, k, packed.data_ptr(), again.data_ptr(), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(scales, again)
    for y_dtype in (torch.float32, torch.bfloat16):
        assert bool(torch.isfinite(pat.pat_op_f8_gemm(packed, again, n, x, y_dtype=y_dtype)).all())


@pytest.mark.parametrize("m", [1, 40, 300])
def test_captured_and_replayed(pat, m):
    w = _x((512, 384), 1, torch.bfloat16).to(DEV)
    pw = pat.pat_op_f8_pack_weight(w)
    x, y = _x((m, 384), 2).to(DEV), torch.empty(m, 512, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        pat.pat_op_f8_gemm(*pw, 512, x, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        pat.pat_op_f8_gemm(*pw, 512, x, y)
    for i in range(3):
        x.copy_(_x((m, 384), 10 + i))
        y.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        eager = pat.pat_op_f8_gemm(*pw, 512, x)
        assert torch.equal(y, eager)


def test_same_call_twice_is_the_same_bits(pat):
    for m in (1, 24, 130, 700):
        x, w = _x((m, 2048), 1).to(DEV), _x((1000, 2048), 2, torch.bfloat16).to(DEV)
        pw = pat.pat_op_f8_pack_weight(w)
        assert torch.equal(pat.pat_op_f8_gemm(*pw, 1000, x), pat.pat_op_f8_gemm(*pw, 1000, x))
