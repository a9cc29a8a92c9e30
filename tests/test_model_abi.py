"""include/detonation_model.h: every declared symbol is exported, the header is plain C, and the host-side checks
refuse what the kernels do not take (these calls return before any launch)."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

from paper_2502_06728_amd import binding, model_ops as ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, NULL, BAD, UNSUPPORTED, ALIGN = 0, 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2502_06728_amd import build
        build.build()
    return ops._load()


def rows(data=4096, ld=64, dtype=0, reserved=0):
    return ctypes.byref(ops.deto_rows(data, ld, dtype, reserved))


def act8(codes=4096, ld=64, exps=4096, ld_exps=2):
    return ctypes.byref(ops.deto_act8(codes, ld, exps, ld_exps))


def norm(pre=1, post=0, eps_pre=1e-6, eps_post=1e-6, scale=1.0, dtype=0, rows_per_gate=0, w_pre=None,
         gate=None, ld_gate=0):
    s = ops.deto_norm_residual(pre, post, eps_pre, eps_post, scale, dtype, rows_per_gate, w_pre)
    s.gate, s.ld_gate = gate, ld_gate
    return ctypes.byref(s)


def test_every_declared_symbol_is_exported(lib):
    text = open(os.path.join(ROOT, "include", "detonation_model.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(detonation_\w+)\s*\(", text))
    assert names == set(ops.EXPORTS)
    for name in names:
        assert getattr(lib, name) is not None


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "detonation_model.h"\n'
                   'int use(void) { deto_rows r = {0, 64, DETO_BF16, 0}; deto_act8 q = {0, 64, 0, 2};\n'
                   '  return detonation_act8_encode(0, 64, &r, &q, 0); }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-fsyntax-only",
                    "-I", os.path.join(ROOT, "include"), str(src)], check=True)


def test_struct_layouts_match_the_header(tmp_path):
    src, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    src.write_text('#include "detonation_model.h"\n#include <stddef.h>\n#include <stdio.h>\n'
                   'int main(void) { printf("%zu %zu %zu %zu %zu %zu", sizeof(deto_rows), '
                   'sizeof(deto_act8), sizeof(deto_norm_residual), sizeof(deto_norm_grads), '
                   'offsetof(deto_norm_residual, rows_per_gate), offsetof(deto_norm_residual, gate)); '
                   'return 0; }\n')
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(ops.deto_rows), ctypes.sizeof(ops.deto_act8),
                   ctypes.sizeof(ops.deto_norm_residual), ctypes.sizeof(ops.deto_norm_grads),
                   ops.deto_norm_residual.rows_per_gate.offset, ops.deto_norm_residual.gate.offset]


def test_logprobs_refusals(lib):
    vp = ctypes.c_void_p

    def f(T=4, V=64, x=rows(), scale=1.0, y=4096, yb=8, logp=4096, top=0, idx=None, ws=4096):
        return lib.detonation_token_logprobs(T, V, x, scale, vp(y), yb, vp(logp), None, None, top,
                                             vp(idx), None, None, vp(ws), None)
    assert f(T=-1) == BAD and f(V=0) == BAD and f(V=1 << 31) == BAD
    assert f(top=33) == BAD and f(top=-1) == BAD and f(V=8, top=9) == BAD
    assert f(scale=0.0) == BAD and f(scale=-1.0) == BAD and f(scale=float("nan")) == BAD
    assert f(scale=float("inf")) == BAD and f(yb=2) == BAD
    assert f(x=None) == NULL and f(x=rows(data=None)) == NULL and f(y=None) == NULL
    assert f(logp=None) == NULL and f(top=4) == NULL
    assert f(V=1 << 16, x=rows(ld=1 << 16), ws=None) == NULL      # pieces to join, no workspace
    assert f(x=rows(dtype=3)) == BAD and f(x=rows(ld=63)) == BAD and f(x=rows(reserved=1)) == BAD
    assert f(x=rows(data=4098)) == ALIGN and f(y=4100) == ALIGN and f(logp=4098) == ALIGN
    assert f(T=0, x=None, y=None, logp=None) == OK
    assert lib.detonation_token_logprobs_workspace(4, 8, 9) == -1
    assert lib.detonation_token_logprobs_workspace(0, 8, 1) >= 0

    def b(T=4, V=64, x=rows(), dx=rows(), scale=1.0, stats=4096, ent=None, g=4096, ge=None):
        return lib.detonation_token_logprobs_backward(T, V, x, scale, vp(4096), 8, vp(stats), vp(ent),
                                                      vp(g), vp(ge), dx, None)
    assert b(T=-1) == BAD and b(scale=0.0) == BAD and b(stats=None) == NULL and b(dx=None) == NULL
    assert b(g=None) == NULL and b(ge=4096) == NULL and b(dx=rows(dtype=1)) == BAD
    assert b(stats=4098) == ALIGN and b(T=0, x=None, dx=None, stats=None) == OK
    assert b(T=1 << 31, V=1 << 30, x=rows(ld=1 << 30), dx=rows(ld=1 << 30)) == UNSUPPORTED


def test_norm_refusals(lib):
    def f(cfg=norm(), T=4, D=64, x=rows(), f=None, xo=None, y=rows(), y8=None):
        return lib.detonation_norm_residual(cfg, T, D, x, f, xo, y, y8, None)
    assert f(cfg=None) == NULL and f(T=-1) == BAD and f(D=0) == BAD and f(D=16385) == UNSUPPORTED
    assert f(cfg=norm(pre=3)) == BAD and f(cfg=norm(post=-1)) == BAD and f(cfg=norm(dtype=3)) == BAD
    assert f(cfg=norm(eps_pre=-1.0)) == BAD and f(cfg=norm(eps_post=float("nan"))) == BAD
    assert f(cfg=norm(scale=float("inf"))) == BAD and f(cfg=norm(rows_per_gate=-1)) == BAD
    assert f(x=None) == NULL and f(y=None) == NULL
    assert f(xo=rows()) == BAD                                   # nothing to add
    assert f(cfg=norm(post=1)) == BAD and f(cfg=norm(gate=4096)) == BAD
    assert f(f=rows()) == NULL                                   # a branch, but no x_out
    assert f(cfg=norm(pre=0), y=None) == BAD                     # nothing at all
    assert f(cfg=norm(pre=0), f=rows(), xo=rows()) == BAD        # y without a norm
    assert f(f=rows(dtype=1), xo=rows()) == BAD                  # y is not of f's type
    assert f(x=rows(dtype=1), f=rows(dtype=2), xo=rows(dtype=1), y=rows(dtype=2)) == BAD
    assert f(x=rows(dtype=1), xo=rows(), f=rows(dtype=1), y=rows(dtype=1)) == BAD
    assert f(cfg=norm(w_pre=4098)) == ALIGN and f(x=rows(data=4098)) == ALIGN
    assert f(y8=act8(exps=None)) == NULL and f(y8=act8(ld_exps=1)) == BAD
    assert f(cfg=norm(gate=4096, rows_per_gate=2, ld_gate=63), f=rows(), xo=rows()) == BAD
    assert f(T=0, x=None, y=None) == OK
    assert lib.detonation_norm_residual_workspace(norm(), 4, 16385) == -1
    assert lib.detonation_norm_residual_workspace(None, 4, 64) == -1

    def grads(**kw):
        return ctypes.byref(ops.deto_norm_grads(**kw))

    def b(cfg=norm(), T=4, D=64, x=rows(), f=None, dy=rows(), dxo=None, dx=rows(), df=None, g=None,
          ws=None):
        return lib.detonation_norm_residual_backward(cfg, T, D, x, f, dy, dxo, dx, df, g,
                                                     ctypes.c_void_p(ws), None)
    assert b(cfg=None) == NULL and b(x=None) == NULL and b(dy=None) == NULL and b(dx=None) == NULL
    assert b(f=rows()) == NULL and b(df=rows()) == BAD           # df iff f
    assert b(g=grads(w_post=4096)) == BAD and b(g=grads(gate=4096)) == BAD
    assert b(cfg=norm(pre=0, post=1), f=rows(), df=rows(), dy=None, g=grads(w_pre=4096)) == BAD
    assert b(g=grads(w_pre=4096)) == NULL                        # no workspace
    assert b(g=grads(w_pre=4098), ws=4096) == ALIGN and b(g=grads(w_pre=4096), ws=4100) == ALIGN
    assert b(dxo=rows(dtype=1)) == BAD and b(dx=rows(dtype=1)) == BAD
    assert b(T=0, x=None, dy=None, dx=None) == OK


def test_act8_refusals(lib):
    e, d = lib.detonation_act8_encode, lib.detonation_act8_decode
    for f in (lambda T=4, D=64, x=rows(), q=act8(): e(T, D, x, q, None),
              lambda T=4, D=64, x=rows(), q=act8(): d(T, D, q, x, None)):
        assert f(T=-1) == BAD and f(D=0) == BAD and f(D=(1 << 30) + 1) == BAD
        assert f(x=None) == NULL and f(q=None) == NULL and f(q=act8(exps=None)) == NULL
        assert f(q=act8(codes=None)) == NULL and f(q=act8(ld=63)) == BAD and f(q=act8(ld_exps=1)) == BAD
        assert f(x=rows(dtype=3)) == BAD and f(x=rows(data=4097)) == ALIGN
        assert f(T=0, x=None, q=None) == OK


def test_glu_refusals(lib):
    def f(act=0, T=4, D=64, a=rows(), b=rows(), h=rows(), a8=act8(), b8=act8()):
        return lib.detonation_glu_forward(act, T, D, a, b, h, a8, b8, None)
    assert f(act=4) == BAD and f(act=-1) == BAD and f(T=-1) == BAD and f(D=0) == BAD
    assert f(a=None) == NULL and f(h=None) == NULL and f(b=None) == BAD     # b8 of nothing
    assert f(b=rows(dtype=1)) == BAD and f(h=rows(dtype=1)) == BAD and f(a8=act8(ld=1)) == BAD
    assert f(T=0, a=None, h=None) == OK

    def g(act=0, T=4, D=64, dh=rows(), a8=act8(), b8=act8(), da=rows(), db=rows(), h8=None):
        return lib.detonation_glu_backward(act, T, D, dh, a8, b8, da, db, h8, None)
    assert g(act=9) == BAD and g(dh=None) == NULL and g(a8=None) == NULL and g(da=None) == NULL
    assert g(db=None) == NULL and g(b8=None) == BAD and g(da=rows(dtype=2)) == BAD
    assert g(h8=act8(ld_exps=1)) == BAD and g(T=0, dh=None, a8=None, da=None) == OK


def test_weight_grad_refusals(lib):
    def f(T=4, N=64, K=64, dy=rows(), x=act8(), dw=rows(), ws=4096):
        return lib.detonation_act8_weight_grad(T, N, K, dy, x, dw, 0, ctypes.c_void_p(ws), None)
    assert f(T=-1) == BAD and f(N=0) == BAD and f(K=0) == BAD and f(T=(1 << 30) + 1) == BAD
    assert f(dw=None) == NULL and f(dy=None) == NULL and f(x=None) == NULL
    assert f(dy=rows(dtype=3)) == BAD and f(dw=rows(ld=63)) == BAD and f(x=act8(ld=63)) == BAD
    assert f(dy=rows(data=4097, dtype=1)) == ALIGN
    assert f(T=4096, ws=None) == NULL and f(T=4096, ws=4100) == ALIGN
    assert lib.detonation_act8_weight_grad_workspace(4, 0, 4) == -1
    assert lib.detonation_act8_weight_grad_workspace(4096, 64, 64) > 0


def test_weight_grad_sizes_whose_sums_would_not_be_counted(lib):
    ws, big = lib.detonation_act8_weight_grad_workspace, 1 << 30
    assert ws(64, big, big) == -1 and ws(64, 1 << 20, (1 << 20) + 1) == -1 and ws(big + 1, 8, 8) == -1
    assert lib.detonation_act8_weight_grad(4, big, big, rows(ld=big), act8(ld=big, ld_exps=big), rows(ld=big), 0,
                                           None, None) == BAD


def test_binding_refuses_host_tensors():
    x, y = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="device"):
        ops.detonation_token_logprobs(x, y, torch.zeros(4))
    with pytest.raises(ValueError, match="device"):
        ops.detonation_act8_encode(x, ops.Act8(torch.zeros(4, 64, dtype=torch.int8),
                                               torch.zeros(4, 2, dtype=torch.uint8)))
    with pytest.raises(ValueError, match="device"):
        ops.detonation_norm_residual(ops.NormResidual(), x, None, None, x)
    with pytest.raises(ValueError):
        ops.token_logprobs_workspace(4, 8, 33)
    with pytest.raises(ValueError):
        ops.act8_weight_grad_workspace(4, 0, 3)
