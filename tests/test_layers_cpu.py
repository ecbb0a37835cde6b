"""Norms and embedding on a host without a GPU: sizes, and refusals that come before any CUDA call."""
import os
import subprocess

import pytest
import torch

FAKE = 4096  # never dereferenced: the checks are host-only
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def meq():
    from paper_2609_35701_gb300 import build

    build.build()
    from paper_2609_35701_gb300 import meq as m

    return m


def _refused(meq, fn, base, cases):
    for kw, text in cases:
        assert fn(*dict(base, **kw).values()) == 1, kw
        assert text in meq.lib.meq_last_error(None), (kw, meq.lib.meq_last_error(None))


def test_norm_refusals(meq):
    base = dict(x=FAKE, ld_x=8, residual=None, ld_residual=0, type=F32, rows=4, cols=8, weight=FAKE, bias=None, weight_type=F32, eps=1e-5, y=FAKE,
                ld_y=8, h=None, ld_h=0, mean=FAKE, rstd=FAKE, stream=None)
    _refused(meq, meq.lib.meq_layer_norm, base, [
        (dict(type=3), b"meq_dtype"), (dict(weight_type=-1), b"meq_dtype"), (dict(rows=-1), b"rows"), (dict(rows=(1 << 27) + 1), b"rows"),
        (dict(cols=0), b"cols"), (dict(cols=(1 << 20) + 1, ld_x=1 << 21, ld_y=1 << 21), b"cols"), (dict(ld_x=7), b"stride of x"),
        (dict(ld_y=7), b"stride of y"), (dict(residual=FAKE, ld_residual=7, h=2 * FAKE, ld_h=8), b"stride of residual"),
        (dict(residual=FAKE, ld_residual=8, h=2 * FAKE, ld_h=7), b"stride of h"), (dict(x=None), b"x must not"), (dict(y=None), b"y must not"),
        (dict(residual=FAKE, ld_residual=8), b"h must not"), (dict(h=2 * FAKE, ld_h=8), b"residual only"),
        (dict(residual=FAKE, ld_residual=8, h=FAKE, ld_h=8), b"the same"), (dict(eps=0.0), b"eps"), (dict(eps=float("nan")), b"eps"),
        (dict(eps=float("inf")), b"eps"), (dict(rstd=None), b"rstd"), (dict(x=FAKE + 2), b"aligned"), (dict(weight=FAKE + 2), b"aligned"),
        (dict(bias=FAKE + 1, weight_type=BF16), b"aligned"), (dict(mean=FAKE + 2), b"aligned"), (dict(ld_x=1 << 41), b"stride of x")])
    base = dict(dy=FAKE, ld_dy=8, h=FAKE, ld_h=8, dh=None, ld_dh=0, type=F32, rows=4, cols=8, weight=FAKE, weight_type=F32, mean=FAKE, rstd=FAKE, dx=FAKE,
                ld_dx=8, dweight=FAKE, dbias=FAKE, grad_type=F32, work=FAKE, stream=None)
    _refused(meq, meq.lib.meq_layer_norm_grad, base, [
        (dict(type=5), b"meq_dtype"), (dict(grad_type=3), b"meq_dtype"), (dict(rows=-2), b"rows"), (dict(cols=0), b"cols"), (dict(ld_dy=1), b"stride of dy"),
        (dict(ld_h=1), b"stride of h"), (dict(dh=FAKE, ld_dh=1), b"stride of dh"), (dict(ld_dx=1), b"stride of dx"), (dict(dy=None), b"dy must not"),
        (dict(h=None), b"h must not"), (dict(dx=None), b"dx must not"), (dict(rstd=None), b"rstd"), (dict(work=None, rows=9000), b"work"), (dict(work=FAKE + 4), b"work"),
        (dict(dweight=FAKE + 2), b"aligned"), (dict(dbias=FAKE + 1, grad_type=BF16), b"aligned"), (dict(dx=FAKE + 1, type=BF16), b"aligned")])
    assert meq.lib.meq_layer_norm(None, 8, None, 0, F32, 0, 8, None, None, F32, 1e-5, None, 8, None, 0, None, None, None) == 0
    assert meq.lib.meq_layer_norm_grad(None, 8, None, 8, None, 0, F32, 0, 8, None, F32, None, None, None, 8, None, None, F32, FAKE, None) == 0
    assert meq.lib.meq_layer_norm_work_floats(-1, 8) == 0 and meq.lib.meq_layer_norm_work_floats(10, 8) >= 2 * 8


def test_embedding_refusals(meq):
    base = dict(tokens=FAKE, n=4, table=FAKE, table_type=F32, vocab=10, cols=8, ld_table=8, scale=1.0, out=FAKE, out_type=F32, ld_out=8, stream=None)
    _refused(meq, meq.lib.meq_embedding, base, [
        (dict(table_type=3), b"meq_dtype"), (dict(out_type=-1), b"meq_dtype"), (dict(n=-1), b"n must"), (dict(n=(1 << 27) + 1), b"n must"),
        (dict(vocab=0), b"vocab"), (dict(vocab=(1 << 28) + 1), b"vocab"), (dict(cols=0), b"cols"), (dict(cols=(1 << 20) + 1), b"cols"),
        (dict(ld_table=7), b"strides"), (dict(ld_out=7), b"strides"), (dict(ld_out=1 << 35), b"strides"), (dict(tokens=None), b"NULL"),
        (dict(table=None), b"NULL"), (dict(out=None), b"NULL"), (dict(tokens=FAKE + 4), b"aligned"), (dict(table=FAKE + 2), b"aligned"),
        (dict(out=FAKE + 1, out_type=BF16), b"aligned")])
    assert meq.lib.meq_embedding(None, 0, None, F32, 10, 8, 8, 1.0, None, F32, 8, None) == 0
    base = dict(grad=FAKE, type=F32, n=4, cols=8, ld=8, tokens=FAKE, vocab=10, scale=1.0, out=FAKE, out_type=F32, ld_out=8, accumulate=0, work=FAKE,
                stream=None)
    _refused(meq, meq.lib.meq_embedding_grad, base, [
        (dict(type=3), b"meq_dtype"), (dict(out_type=7), b"meq_dtype"), (dict(n=-1), b"n must"), (dict(vocab=0), b"vocab"), (dict(cols=0), b"cols"),
        (dict(ld=7), b"strides"), (dict(ld_out=7), b"strides"), (dict(grad=None), b"NULL"), (dict(tokens=None), b"NULL"), (dict(out=None), b"NULL"),
        (dict(work=None), b"work"), (dict(work=FAKE + 8), b"work"), (dict(grad=FAKE + 2), b"aligned"), (dict(out=FAKE + 2), b"aligned")])
    assert meq.lib.meq_embedding_grad(None, F32, 0, 8, 8, None, 10, 1.0, FAKE, F32, 8, 1, FAKE, None) == 0   # nothing to add
    assert meq.lib.meq_embedding_work_floats(-1, 9, 8) == 0 and meq.lib.meq_embedding_work_floats(1000, 9, 8) >= 4 * 1000


def test_binding_refuses_host_tensors(meq):
    x, w, v, t = torch.zeros(4, 8), torch.ones(8), torch.zeros(4), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: meq.layer_norm(x, w), lambda: meq.rms_norm(x, w), lambda: meq.layer_norm_grad(x, x, w, v, v), lambda: meq.rms_norm_grad(x, x, w, v),
                 lambda: meq.embedding(t, x), lambda: meq.embedding_grad(x, t, x)):
        with pytest.raises(ValueError):
            call()


SORT_BLOCKS = """
#include <cstdio>
#include "embedding_sort.cuh"
int main() {
  const long long tokens[] = {0, 256, 257, 16384, 16385, 1 << 27};
  const int held[][2] = {{14, 7}, {1, 1}, {3, 0}, {0, 0}};  // clusters of 8 and of 16 blocks that a device holds
  for (const auto& device : held)
    for (long long n : tokens) {
      int asked = 0, clusters = -1;
      const int blocks = meq::sort_blocks(n, [&](int b) { ++asked; return device[b == 16]; }, &clusters);
      std::printf("%d,%d,%d ", blocks, clusters, asked);
    }
}
"""


def test_the_sorts_cluster_is_one_that_the_device_holds(tmp_path):
    """16 blocks sort many tokens where they can be had, else 8; few tokens ask for no cluster."""
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_35701_gb300", "csrc")
    (tmp_path / "blocks.cpp").write_text(SORT_BLOCKS)
    exe = str(tmp_path / "blocks")
    subprocess.run(["g++", "-std=c++17", "-I", csrc, str(tmp_path / "blocks.cpp"), "-o", exe], check=True)
    none = ["0,0,0"] * 2
    want = (none + ["8,14,1"] * 2 + ["16,7,1"] * 2) + (none + ["8,1,1"] * 2 + ["16,1,1"] * 2) + (none + ["8,3,1"] * 2 + ["8,3,2"] * 2)
    want += none + ["8,0,1"] * 2 + ["8,0,2"] * 2
    assert subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split() == want
