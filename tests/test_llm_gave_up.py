"""What a kernel makes of another kernel's results where that one gave up a bounded wait: nothing, and what is there stays.

No wait runs out here.  The kernels that come second are built from their sources and launched on results that are marked as the first
kernel would mark them."""

import ctypes
import os
import subprocess

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2308_15164_b200", "csrc")
MARK = 0x7FD5A5A5

JOIN = """
extern "C" int t_join(float* part, int rest, int splits, int M, int N, float* out, int ld, int accumulate, int wide) {
    LinArgs a{};
    a.M = M; a.N = N; a.tiles_m = (M + kTM - 1) / kTM; a.tiles_n = (N + kTN - 1) / kTN; a.rest = rest; a.splits = splits; a.part = part;
    a.out = out; a.ld = ld; a.accumulate = accumulate; a.join = 1; a.wide = wide;
    const cudaError_t e = launch_kernel(k_linear_join<kWgrad, ABS_ACT_NONE, float>, rest * kTM / 8, 256, 0, (cudaStream_t)0, false, a);
    return (int)(e != cudaSuccess ? e : cudaDeviceSynchronize());
}
"""
ROWS = """
extern "C" int t_rows(const float* x, const float* g, float* y, float* last, int T, int D, int segs, void* maps, int* status) {
    RecArgs a{};
    a.x = x; a.ld_x = D; a.g = g; a.ld_g = D; a.out = y; a.ld_out = D; a.after = last; a.T = T; a.D = D; a.seqs = 1;
    a.strips = (D + kCols - 1) / kCols; a.segs = segs; a.rows = kTileOf<float, false, false>; a.parts = 1; a.part_rows = a.rows; a.pairs = 1;
    a.maps = static_cast<Map*>(maps);
    const CUtensorMap none{};
    cudaError_t e = launch_kernel(k_recurrence<float, ABS_RECURRENCE_ADD, false, false, false>, a.segs * a.strips, kWarps * 32, smem_bytes<false, false>(false),
                                  (cudaStream_t)0, false, a, none, none, none, none);
    return (int)(e != cudaSuccess ? e : take_status(status, 0));
}
extern "C" int t_tile() { return kTileOf<float, false, false>; }
"""
COLUMNS = """
extern "C" int t_columns(const float* part, int n, int D, float* first, float* second, int accumulate) {
    const cudaError_t e = launch_kernel(k_column_sums, dim3((D + 31) / 32, 2), 1024, 0, (cudaStream_t)0, false, part, n, D, first, second, (float*)nullptr,
                                        (const float*)nullptr, (const float*)nullptr, accumulate);
    return (int)(e != cudaSuccess ? e : cudaDeviceSynchronize());
}
"""


def build(where, name, cut, calls, inside):
    """The kernels of a source file, up to the line that starts with `cut` (inside: of its unnamed namespace), with these functions behind them."""
    text = open(os.path.join(CSRC, name)).read()
    at = text.index(cut)
    source = os.path.join(where, name)
    with open(source, "w") as f:
        f.write(text[:at] + ("}\n" if inside else "namespace abs_sgd {\n") + calls + "}\n")
    lib = source.replace(".cu", ".so")
    subprocess.run([os.environ.get("NVCC", "nvcc"), "-gencode", "arch=compute_100a,code=sm_100a", "-O1", "-std=c++17", "-shared", "-Xcompiler", "-fPIC", "-I",
                    os.path.join(ROOT, "include"), "-I", CSRC, "-o", lib, source], check=True, stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    return ctypes.CDLL(lib)


def ptr(t):
    return ctypes.c_void_p(t.data_ptr())


@pytest.mark.parametrize("wide,N", [(16, 256), (0, 300), (16, 512)])
def test_cut_tiles_of_which_a_part_is_missing(tmp_path_factory, wide, N):
    lib = join_lib(tmp_path_factory)
    M, splits = 256, 3
    rest = (N + 255) // 256
    part = torch.ones(splits, rest, 256, 256, device=DEV)
    for acc in (0, 1):
        def call(p):
            out = torch.full((M, N), 5.0, device=DEV)
            assert lib.t_join(ptr(p), rest, splits, M, N, ptr(out), N, acc, wide) == 0
            return out

        assert (call(part) == splits + 5 * acc).all()
        for k in range(splits):                                  # 32 rows and 64 columns of a part
            p = part.clone()
            p.view(torch.int32)[k, rest - 1, 32:64, :64] = MARK
            out, c = call(p), (rest - 1) * 256
            missing = torch.zeros(M, N, dtype=torch.bool, device=DEV)
            missing[32:64, c:c + 64] = True
            assert (out[missing] == 5).all() and (out[~missing] == splits + 5 * acc).all()
        p = part.clone()
        p[1, 0, 3, 7] = float("nan")                             # a NaN that was computed is none of that
        out = call(p)
        assert out[3, 7].isnan() and int(out.isnan().sum()) == 1


_libs = {}


def join_lib(factory):
    if "join" not in _libs:
        _libs["join"] = build(str(factory.mktemp("join")), "llm_linear.cu", "// The product and its epilogue;", JOIN, True)
    return _libs["join"]


def test_rows_behind_a_segment_whose_map_is_missing(tmp_path):
    lib = build(str(tmp_path), "llm_recurrence.cu", "template <int N>\nint launch_scan(", ROWS, True)
    tile, segs, D = lib.t_tile(), 3, 192
    T = tile * segs
    g = torch.zeros(T, D, device=DEV)                            # gates of one half
    x = torch.ones(T, D, device=DEV)
    maps = torch.zeros(segs - 1, 3, 32, 4, device=DEV)           # [segment][strip][lane]: A, A, B, B
    maps[..., 2:] = 2.0                                          # each leaves a state of 2, as the rows do
    for bad in (None, 0, 1):                                     # the segment of the middle strip that is missing
        m = maps.clone()
        if bad is not None:
            m.view(torch.int32)[bad, 1, :, :2] = MARK
        y, last, status = torch.full((T, D), 7.0, device=DEV), torch.full((1, D), 7.0, device=DEV), ctypes.c_int(0)
        assert lib.t_rows(ptr(x), ptr(g), ptr(y), ptr(last), T, D, segs, ptr(m), ctypes.byref(status)) == 0
        want = torch.full((T, D), 2.0, device=DEV)
        row = torch.arange(tile, device=DEV)
        want[:tile] = (2.0 - 0.5 ** row.double()).float()[:, None]           # from a state of 0: 1, 1.5, 1.75 ...
        end = torch.full((1, D), 2.0, device=DEV)
        if bad is not None:
            want[(bad + 1) * tile:, 64:128] = 7.0
            end[:, 64:128] = 7.0
        assert torch.allclose(y, want, rtol=1e-6, atol=0) and torch.allclose(last, end, rtol=1e-6, atol=0)
        assert (status.value != 0) == (bad is not None)


@pytest.mark.parametrize("n,D", [(1, 5), (40, 33), (700, 64)])
def test_column_sums_of_which_a_part_is_missing(tmp_path_factory, n, D):
    if "columns" not in _libs:
        _libs["columns"] = build(str(tmp_path_factory.mktemp("columns")), "llm_norm.cu", "namespace abs_sgd {\ncudaError_t take_status_norm(", COLUMNS, False)
    lib = _libs["columns"]
    W = (D + 3) // 4 * 4
    part = torch.ones(n, 2, W, device=DEV)
    for acc in (0, 1):
        a, b = torch.full((D,), 5.0, device=DEV), torch.full((D,), 5.0, device=DEV)
        assert lib.t_columns(ptr(part), n, D, ptr(a), ptr(b), acc) == 0
        assert (a == n + 5 * acc).all() and (b == n + 5 * acc).all()
        for row in (0, n // 2, n - 1):
            p = part.clone()
            p.view(torch.int32)[row] = MARK
            a.fill_(5.0), b.fill_(5.0)
            assert lib.t_columns(ptr(p), n, D, ptr(a), ptr(b), acc) == 0
            assert (a == 5).all() and (b == 5).all()
        p = part.clone()
        p[0, 0, D - 1] = float("nan")                            # a NaN that was computed is none of that
        a.fill_(5.0)
        assert lib.t_columns(ptr(p), n, D, ptr(a), ptr(b), acc) == 0
        assert a[D - 1].isnan() and (a[:D - 1] == n + 5 * acc).all()
