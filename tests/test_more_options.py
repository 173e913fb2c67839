"""What the entry points of routing by scores, dense products and the gradients' norm take: checked before any device is asked for, and
how the binding lays it out (no GPU needed)."""
import os
import shutil
import struct
import subprocess

import pytest

from paper_2505_15511_amd import _build, binding as b

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, TOO_LARGE = -1, -4
P = 1 << 12   # an address that nothing looks at


@pytest.fixture(scope="module")
def lib():
    if _build.is_stale():
        _build.build_library()
    return b.load_library()


def _route(lib, n=10, experts=8, k=2, dtype=0, workspace=P, **more):
    f = dict(size=b.SCORING.size, score=1, normalize=1, groups=1, top_groups=1, group_best=1, bias=0, scale=1.0)
    f.update(more)
    scoring = b.SCORING.pack(*f.values())
    back = lib.nomad_route_scored_gradient(P, dtype, n, experts, experts, k, scoring, P, P, P, P, 1 << 20, None)   # (a device that is not there)
    return lib.nomad_route_scored(P, dtype, n, experts, experts, k, scoring, P, P, P, P, P, workspace, 1 << 30, 1 << 20, None), back


def test_scoring(lib):
    for more in ({}, dict(score=0), dict(normalize=0), dict(groups=4, top_groups=1), dict(groups=8, top_groups=2, group_best=2), dict(scale=-2.5), dict(n=0), dict(experts=128, groups=64, top_groups=3)):
        assert all(rc not in (INVALID, TOO_LARGE) for rc in _route(lib, **more)), more
    for more in (dict(size=b.SCORING.size - 8), dict(score=2), dict(normalize=2), dict(groups=3), dict(groups=0), dict(groups=2, top_groups=3), dict(top_groups=0),
                 dict(group_best=3), dict(group_best=0), dict(scale=0.0), dict(scale=1e-39), dict(scale=float("nan")), dict(scale=float("inf")), dict(groups=8, top_groups=1), dict(k=9), dict(k=0), dict(dtype=3), dict(n=-1),
                 dict(experts=130, groups=65)):
        assert _route(lib, **more) == (INVALID, INVALID), more
    assert _route(lib, experts=16385) == (TOO_LARGE, TOO_LARGE) and _route(lib, n=1 << 31) == (TOO_LARGE, TOO_LARGE)
    assert _route(lib, n=100_000, workspace=None)[0] == INVALID


def test_balance(lib):
    assert lib.nomad_balance_bias(P, P, 8, 0.1, P, 1 << 20, None) not in (INVALID, TOO_LARGE)
    for args in ((None, P, 8, 0.1, P), (P, None, 8, 0.1, P), (P, P, 8, 0.1, None), (P, P, 0, 0.1, P), (P, P, 8, float("inf"), P)):
        assert lib.nomad_balance_bias(*args, 1 << 20, None) == INVALID
    assert lib.nomad_balance_bias(P, P, 16385, 0.1, P, 1 << 20, None) == TOO_LARGE


def _product(lib, **more):
    f = dict(size=b.DENSE_ARGS.size, dtype=0, out_dtype=0, activation=0, inner=8, out=4, rows=10, x=P, x_stride=8, w=P, wo=8, wi=1, bias=0, residual=0, rs=0, slope=0, ss=0,
             y=P, ys=4, z=0, zs=4, work=P, bytes=1 << 40, stream=0, device=1 << 20)
    f.update(more)
    return lib.nomad_dense_product(b.DENSE_ARGS.pack(*f.values()))


def test_product(lib):
    for more in ({}, dict(dtype=1, out_dtype=0), dict(dtype=2, out_dtype=2), dict(activation=3), dict(wo=1, wi=4), dict(residual=P, rs=0), dict(residual=P, rs=9), dict(slope=P, ss=4), dict(z=P),
                 dict(rows=1, ys=0), dict(inner=1, wi=7)):
        assert _product(lib, **more) not in (INVALID, TOO_LARGE), more
    assert _product(lib, rows=0, x=0, y=0) == 0
    for more in (dict(size=b.DENSE_ARGS.size - 8), dict(dtype=3), dict(dtype=1, out_dtype=2), dict(out_dtype=1), dict(activation=4), dict(inner=0), dict(out=0), dict(rows=-1), dict(x=0), dict(w=0),
                 dict(y=0), dict(wo=9, wi=2), dict(ys=3), dict(z=P, zs=3), dict(slope=P, bias=P), dict(slope=P, residual=P), dict(slope=P, z=P), dict(x_stride=-1), dict(rs=-1, residual=P)):
        assert _product(lib, **more) == INVALID, more
    for more in (dict(rows=1 << 31), dict(inner=(1 << 20) + 1, wo=1 << 21), dict(out=(1 << 20) + 1, ys=1 << 21)):
        assert _product(lib, **more) == TOO_LARGE, more
    need = lib.nomad_dense_workspace(500, 8192, 768, 1)
    assert need > 0
    long = dict(dtype=1, out_dtype=1, rows=500, inner=8192, out=768, x_stride=8192, wo=8192, ys=768)
    assert _product(lib, **long, bytes=need) not in (INVALID, TOO_LARGE)
    for more in (dict(bytes=need - 1), dict(work=0), dict(work=P + 8)):
        assert _product(lib, **long, **more) == INVALID, more


def _gradient(lib, **more):
    f = dict(size=b.DENSE_GRADIENT_ARGS.size, dtype=0, out_dtype=0, activation=0, inner=8, out=4, rows=10, dy=P, dys=4, z=0, zs=0, x=P, xs=8, w=P, wo=8, wi=1, dx=P, dxs=8, dw=P, db=P,
             work=P, bytes=1 << 40, stream=0, device=1 << 20)
    f.update(more)
    return lib.nomad_dense_gradient(b.DENSE_GRADIENT_ARGS.pack(*f.values()))


def test_gradient(lib):
    for more in ({}, dict(activation=2, z=P, zs=4), dict(dx=0), dict(dw=0, db=0), dict(db=0), dict(dx=0, w=0), dict(rows=0, dy=0, x=0, w=0), dict(dtype=1, out_dtype=0), dict(wo=1, wi=4)):
        assert _gradient(lib, **more) not in (INVALID, TOO_LARGE), more
    for more in (dict(size=8), dict(activation=2), dict(dx=0, dw=0, db=0), dict(dw=0), dict(dxs=7), dict(dy=0), dict(x=0), dict(w=0), dict(wo=9, wi=2), dict(dtype=1, out_dtype=2), dict(rows=-1),
                 dict(activation=2, z=P, zs=4, work=0), dict(dys=-1)):
        assert _gradient(lib, **more) == INVALID, more
    assert _gradient(lib, rows=1 << 31) == TOO_LARGE


def _norm(lib, tensors=((P, 10, 0),), most=1.0, norm=P, bytes=1 << 20, work=P):
    packed = b"".join(b.GRADIENT.pack(*t) for t in tensors)
    return lib.nomad_gradient_norm(packed, len(tensors), most, None, norm, P, work, bytes, 1 << 20, None)


def test_norm(lib):
    assert _norm(lib) not in (INVALID, TOO_LARGE) and _norm(lib, most=float("inf")) not in (INVALID, TOO_LARGE)
    assert _norm(lib, tensors=((P, 10, 1), (0, 0, 2), (P + 2, 3, 1))) not in (INVALID, TOO_LARGE)
    for more in (dict(most=-1.0), dict(most=float("nan")), dict(norm=None), dict(work=None), dict(work=P + 4), dict(bytes=lib.nomad_gradient_norm_workspace(1) - 1), dict(tensors=((0, 10, 0),)),
                 dict(tensors=((P, -1, 0),)), dict(tensors=((P, 10, 3),)), dict(tensors=((P + 2, 10, 0),)), dict(tensors=((P + 1, 10, 1),))):
        assert _norm(lib, **more) == INVALID, more
    assert _norm(lib, tensors=((P, 1 << 51, 0),)) == TOO_LARGE


LAYOUT = r"""
#include <stdio.h>
#include <stddef.h>
#include "nomad.h"
int main(void) {
    printf("%zu %zu %zu %zu\n", sizeof(nomad_scoring), sizeof(nomad_dense_args), sizeof(nomad_dense_gradient_args), sizeof(nomad_gradient));
    printf("%zu %zu %zu %zu\n", offsetof(nomad_scoring, bias), offsetof(nomad_scoring, scale), offsetof(nomad_dense_args, rows), offsetof(nomad_dense_args, residual));
    printf("%zu %zu %zu %zu\n", offsetof(nomad_dense_args, workspace), offsetof(nomad_dense_args, device), offsetof(nomad_dense_gradient_args, w), offsetof(nomad_dense_gradient_args, db));
    printf("%zu %zu\n", offsetof(nomad_dense_gradient_args, device), offsetof(nomad_gradient, dtype));
    return 0;
}
"""


def test_argument_layouts(tmp_path):
    """What the binding packs is what the header declares."""
    if not shutil.which("gcc"):
        pytest.skip("no C compiler")
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text(LAYOUT)
    subprocess.run(["gcc", "-std=c99", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    said = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]

    def at(fmt, part):                                         # offset of the field behind the first `part` of a format
        return struct.calcsize("@" + part + "0" + fmt)
    assert said[:4] == [b.SCORING.size, b.DENSE_ARGS.size, b.DENSE_GRADIENT_ARGS.size, b.GRADIENT.size]
    assert said[4:8] == [at("P", "I5i"), at("f", "I5iP"), at("q", "I5i"), at("P", "I5iqPqPqqP")]
    assert said[8:12] == [at("P", "I5iqPqPqqPPqPqPqPq"), at("i", "I5iqPqPqqPPqPqPqPqPqP"), at("P", "I5iqPqPqPq"), at("P", "I5iqPqPqPqPqqPqP")]
    assert said[12:] == [at("i", "I5iqPqPqPqPqqPqPPPqP"), at("i", "Pq")]
