"""A cluster that shares a tile's K writes one slice of sums: an epilogue that stores to a slice a split, as the sum
over pieces does, gets split 0 from every CTA.  Built from a few lines of its own, since the sizes of the
calls never choose clusters for such sums."""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from paper_2407_11698_gb300 import build as nbuild

SOURCE = r'''
#include "head_gemm.cuh"
using namespace nitro;
namespace nitro { namespace {
struct EpiSlice {
    static constexpr bool kFold = false, kTail = false;
    struct Args { float* c; int64_t ldc, slice; };
    const Args& a; const HgArgs& g; const HgPart& p; float* base;
    __device__ EpiSlice(const Args& a_, const HgArgs& g_, const HgTile& t, const HgPart& p_)
        : a(a_), g(g_), p(p_), base(a_.c + t.split * a_.slice) {}
    __device__ void fetch(int) {}
    __device__ void cols(int c, float* v) {
        for (int j = 0; j < 32; ++j)
            if (p.row < p.rows && p.col0 + c + j < g.N) base[(int64_t)p.row * a.ldc + p.col0 + c + j] = v[j];
    }
    __device__ void done() {}
};
template <int KS>
int run(const HgProblem& p, const HgOperand& a, const HgOperand& b, const EpiSlice::Args& e, cudaStream_t s) {
    return hg_launch_as<EpiSlice, 1, 128, false, false, false, 1, 1, KS>(KS, p, a, b, e, s) != cudaSuccess;
}
} }
extern "C" int cluster_product(const void* a, const void* b, int m, int n, int k, float* c, int64_t slice, uint32_t* status, int ks,
                               void* stream) {
    HgProblem p{m, n, k};
    p.status = status;
    const HgOperand oa{a, k, m, k, 1, 0}, ob{b, k, n, k, 1, 0};
    const EpiSlice::Args e{c, n, slice};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return ks == 2 ? run<2>(p, oa, ob, e, s) : ks == 4 ? run<4>(p, oa, ob, e, s) : run<8>(p, oa, ob, e, s);
}
'''


@pytest.fixture(scope="module")
def product(tmp_path_factory):
    d = tmp_path_factory.mktemp("cluster")
    src, so = d / "cluster.cu", d / "cluster.so"
    src.write_text(SOURCE)
    objs = [os.path.join(nbuild.OUT_DIR, "prof.o")]
    subprocess.run([nbuild.nvcc()] + nbuild.ARCH + nbuild.FLAGS + ["-shared", str(src)] + objs + ["-o", str(so)], check=True,
                   capture_output=True, text=True)
    f = ctypes.CDLL(str(so)).cluster_product
    V, I = ctypes.c_void_p, ctypes.c_int
    f.argtypes = [V, V, I, I, I, V, ctypes.c_int64, V, I, V]
    return f


@pytest.mark.parametrize("ks", [2, 4, 8])
@pytest.mark.parametrize("m, n", [(128, 128), (200, 300)])
def test_sums_go_to_one_slice(product, m, n, ks):
    k = 1024
    g = torch.Generator(device="cuda").manual_seed(ks)
    a = torch.randint(-4, 5, (m, k), generator=g, device="cuda").to(torch.bfloat16)
    b = torch.randint(-4, 5, (n, k), generator=g, device="cuda").to(torch.bfloat16)
    c = torch.full((ks, m, n), -7.5, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    assert product(a.data_ptr(), b.data_ptr(), m, n, k, c.data_ptr(), m * n, status.data_ptr(), ks, None) == 0
    torch.cuda.synchronize()
    assert status.item() == 0
    assert torch.equal(c[0].double(), a.double() @ b.double().t())      # integers: exact
    assert (c[1:] == -7.5).all()
