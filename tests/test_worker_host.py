"""The operators of a worker's step through the C-ABI and the binding, without a GPU: the header is C,
its constants are the binding's, and what a kernel could not take is refused before any launch."""
import ctypes
import os
import re
import subprocess

import pytest
import torch

import paper_2010_04902_amd as B
from paper_2010_04902_amd import worker

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, EUNSUPPORTED, ENOMEM = 0, -1, -2, -3
P = 0x10000  # an address nothing reads: every call below returns before a launch


def test_header_is_plain_c_and_agrees_with_the_binding(tmp_path):
    src = tmp_path / "consts.c"
    src.write_text('''#include <stdio.h>
#include "byzshield_worker.h"
int main(void) {
    printf("%d %d %d %d %d %d %d %d %d\\n", BYZ_F32, BYZ_BF16, BYZ_F16, BYZ_ACT_NONE, BYZ_ACT_RELU, BYZ_ACT_SILU,
           BYZ_ACT_GELU, BYZ_ACT_SIGMOID, BYZ_MAX_TEACHER);
    return 0;
}
''')
    exe = tmp_path / "consts"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [B.BYZ_F32, B.BYZ_BF16, B.BYZ_F16, B.BYZ_ACT_NONE, B.BYZ_ACT_RELU, B.BYZ_ACT_SILU, B.BYZ_ACT_GELU,
                   B.BYZ_ACT_SIGMOID, B.BYZ_MAX_TEACHER]


def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "byzshield_worker.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    names = set(re.findall(r"\b(byz_[a-z_0-9]+)\s*\(", header))
    assert len(names) >= 9
    lib = ctypes.CDLL(B.library_path())
    for n in names:
        assert hasattr(lib, n), n


# ------------------------------------------------------------------ C-ABI refusals


def _norm(x=P, xs=64 * 16, xp=16, n=2, p=64, c=16, groups=4, dtype=0, gamma=None, beta=None, eps=1e-5, act=0, y=P,
          ys=64 * 16, yp=16, mean=P, rstd=P, ws=None, nbytes=0):
    return worker._load().byz_group_norm(x, xs, xp, n, p, c, groups, dtype, gamma, beta, eps, act, y, ys, yp, mean, rstd,
                                         ws, nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(y=None), dict(mean=None), dict(rstd=None), dict(n=-1), dict(p=-1), dict(c=0), dict(c=-16),
    dict(groups=0), dict(groups=-4), dict(groups=3), dict(groups=32), dict(dtype=3), dict(dtype=-1), dict(act=5), dict(act=-1),
    dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(xp=15), dict(yp=8), dict(xs=-1), dict(ys=-1),
    dict(ys=64 * 16 - 1), dict(x=P + 2), dict(y=P + 1), dict(n=1 << 40, p=1 << 40), dict(xs=1 << 62), dict(xp=1 << 62)],
    ids=str)
def test_group_norm_refusals(bad):
    assert _norm(**bad) == EINVAL


def test_group_norm_needs_its_workspace():
    # a sample larger than a compute unit's registers is cut into chunks, whose statistics need memory
    big = dict(n=4, p=112 * 112, c=64, groups=32, xs=112 * 112 * 64, xp=64, ys=112 * 112 * 64, yp=64)
    need = worker._load().byz_group_norm_workspace_bytes(4, 112 * 112, 64, 32, 0)
    assert need > 0
    assert _norm(**big) == ENOMEM
    assert _norm(**big, ws=P, nbytes=64) == ENOMEM
    assert worker._load().byz_group_norm_workspace_bytes(4, 16, 64, 3, 0) == 0  # refused sizes need none


def _norm_backward(dy=P, ds=64 * 16, dp=16, x=P, xs=64 * 16, xp=16, n=2, p=64, c=16, groups=4, dtype=0, mean=P, rstd=P,
                   act=0, dx=P, os_=64 * 16, op=16, dgamma=P, dbeta=P, ws=P, nbytes=1 << 30):
    return worker._load().byz_group_norm_backward(dy, ds, dp, x, xs, xp, n, p, c, groups, dtype, None, None, mean, rstd, act,
                                                  dx, os_, op, dgamma, dbeta, ws, nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(dy=None), dict(x=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(dgamma=None), dict(dbeta=None),
    dict(groups=5), dict(dtype=7), dict(act=9), dict(dp=15), dict(op=3), dict(os_=100), dict(dx=P + 2), dict(xs=-16)], ids=str)
def test_group_norm_backward_refusals(bad):
    assert _norm_backward(**bad) == EINVAL


def test_group_norm_backward_needs_its_workspace():
    assert _norm_backward(nbytes=16) == ENOMEM
    assert _norm_backward(ws=None) == ENOMEM
    assert _norm_backward(ws=P + 4) == ENOMEM


def _distill(logits=P, rows=4, vocab=100, ld=100, dtype=0, teacher=P, index=P, k=5, tld=5, temperature=1.0, loss=P, lse=P):
    return worker._load().byz_distill_loss(logits, rows, vocab, ld, dtype, teacher, index, k, tld, temperature, loss, lse, None)


def _distill_step(logits=P, rows=4, vocab=100, ld=100, dtype=0, teacher=P, index=P, k=5, tld=5, dloss=P, temperature=1.0,
                  loss=P, lse=None, out=P, old=100):
    return worker._load().byz_distill_loss_step(logits, rows, vocab, ld, dtype, teacher, index, k, tld, dloss, temperature,
                                                loss, lse, out, old, None, 0, None)


def _distill_backward(dloss=P, logits=P, rows=4, vocab=100, ld=100, dtype=0, teacher=P, index=P, k=5, tld=5, lse=P,
                      temperature=1.0, out=P, old=100):
    return worker._load().byz_distill_loss_backward(dloss, logits, rows, vocab, ld, dtype, teacher, index, k, tld, lse,
                                                    temperature, out, old, None)


SHARED = [dict(logits=None), dict(teacher=None), dict(index=None), dict(rows=-1), dict(vocab=0), dict(vocab=-5),
          dict(vocab=1 << 31, ld=1 << 31), dict(ld=99), dict(ld=1 << 61), dict(dtype=3), dict(k=0), dict(k=1025, tld=1025),
          dict(tld=4), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")),
          dict(temperature=float("inf")), dict(logits=P + 2)]


@pytest.mark.parametrize("bad", SHARED + [dict(loss=None)], ids=str)
def test_distill_refusals(bad):
    assert _distill(**bad) == EINVAL


@pytest.mark.parametrize("bad", SHARED + [dict(dloss=None), dict(out=None), dict(old=99), dict(out=P + 1)], ids=str)
def test_distill_gradient_refusals(bad):
    assert _distill_step(**bad) == EINVAL
    assert _distill_backward(**bad) == EINVAL


def test_distill_step_needs_its_workspace():
    # long rows are held in registers between two kernels of their own
    need = worker._load().byz_distill_loss_step_workspace_bytes(1000, 100000, 5, 1)
    assert need > 0 and worker._load().byz_distill_loss_step_workspace_bytes(1000, 1000, 5, 1) == 0
    assert _distill_step(rows=1000, vocab=100000, ld=100000, old=100000, dtype=1) == ENOMEM


def test_distill_needs_its_outputs():
    assert _distill_step(loss=None) == EINVAL
    assert _distill_backward(lse=None) == EINVAL
    for call in (_distill, _distill_step, _distill_backward):
        assert call(rows=0) == OK  # nothing to do, whatever the pointers are
        assert call(rows=0, logits=None) == OK


def _ffn(x=P, x_ld=32, wg=P, wu=P, w_ld=32, m=4, k=32, n=8, dtype=1, act=2, h=P, h_ld=8, gate=None, up=None, gate_ld=0,
         ws=None, nbytes=0):
    return worker._load().byz_gated_ffn(x, x_ld, wg, wu, w_ld, m, k, n, dtype, act, h, h_ld, gate, up, gate_ld, ws, nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(wg=None), dict(wu=None), dict(h=None), dict(m=-1), dict(k=-1), dict(n=-1), dict(x_ld=31), dict(w_ld=31),
    dict(h_ld=7), dict(dtype=3), dict(act=5), dict(gate=P), dict(up=P), dict(gate=P, up=P, gate_ld=7),
    dict(gate=P + 2, up=P, gate_ld=8), dict(x=P + 1), dict(m=1 << 31), dict(x_ld=1 << 62)], ids=str)
def test_gated_ffn_refusals(bad):
    assert _ffn(**bad) == EINVAL


def test_gated_ffn_types_and_empty_calls():
    assert _ffn(dtype=0) == EUNSUPPORTED
    assert _ffn(m=0) == OK and _ffn(n=0) == OK and _ffn(m=0, x=None, h=None) == OK


def test_gated_ffn_needs_its_workspace():
    # more tokens than the kernel for few takes, rows that do not start at 16-byte boundaries
    need = worker._load().byz_gated_ffn_workspace_bytes(40, 31, 8, 1)
    assert need > 0 and worker._load().byz_gated_ffn_workspace_bytes(16, 31, 8, 1) == 0
    odd = dict(m=40, k=31, x_ld=31, w_ld=31)
    assert _ffn(**odd) == ENOMEM
    assert _ffn(**odd, ws=P, nbytes=need - 1) == ENOMEM
    assert _ffn(**odd, ws=P + 2, nbytes=need) == ENOMEM
    assert _ffn(m=40, x=P + 2) == ENOMEM


def _ffn_backward(dh=P, dh_ld=8, x=P, x_ld=32, wg=P, wu=P, w_ld=32, gate=P, up=P, gate_ld=8, m=4, k=32, n=8, dtype=1, act=2,
                  dx=P, dx_ld=32, dwg=P, dwu=P, dw_ld=32, ws=P, nbytes=1 << 30):
    return worker._load().byz_gated_ffn_backward(dh, dh_ld, x, x_ld, wg, wu, w_ld, gate, up, gate_ld, m, k, n, dtype, act, dx,
                                                 dx_ld, dwg, dwu, dw_ld, ws, nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(dh=None), dict(x=None), dict(wg=None), dict(wu=None), dict(gate=None), dict(up=None), dict(dwg=None), dict(dwu=None),
    dict(dh_ld=7), dict(gate_ld=7), dict(dx_ld=31), dict(dw_ld=31), dict(dtype=4), dict(act=-1), dict(m=-2)], ids=str)
def test_gated_ffn_backward_refusals(bad):
    assert _ffn_backward(**bad) == EINVAL


def test_gated_ffn_backward_needs_its_workspace():
    assert _ffn_backward(dtype=0) == EUNSUPPORTED
    assert _ffn_backward(nbytes=16) == ENOMEM
    assert _ffn_backward(ws=None) == ENOMEM
    assert _ffn_backward(ws=P + 2) == ENOMEM


# ------------------------------------------------------------------ the binding's refusals


def test_binding_refuses_host_tensors():
    x = torch.zeros(2, 8, 4, 4).contiguous(memory_format=torch.channels_last)
    with pytest.raises(ValueError, match="CUDA"):
        B.byz_group_norm(x, 4)
    with pytest.raises(ValueError, match="CUDA"):
        B.byz_group_norm_backward(x, x, 4, torch.zeros(2, 4), torch.zeros(2, 4))
    with pytest.raises(ValueError, match="CUDA"):
        B.byz_distill_loss(torch.zeros(2, 8), torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32))
    w = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        B.byz_gated_ffn(w, w, w)


def test_binding_refuses_layouts_the_kernels_do_not_read():
    with pytest.raises(ValueError, match="channels last"):
        B.byz_group_norm(torch.zeros(2, 8, 4, 4), 4)          # channels first
    with pytest.raises(ValueError, match="channels last"):
        B.byz_group_norm(torch.zeros(2, 8, 16).transpose(1, 2), 4)
    with pytest.raises(ValueError, match="channels last"):
        B.byz_group_norm(torch.zeros(2, 4, 6, 8)[:, :, :4].permute(0, 3, 1, 2)[:, :, ::2], 4)  # every other row
    with pytest.raises(ValueError, match="must be"):
        B.byz_group_norm(torch.zeros(2, 8), 4)
    i = torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="neighbouring"):
        B.byz_distill_loss(torch.zeros(8, 2).t(), torch.zeros(2, 3), i)
    with pytest.raises(ValueError, match="neighbouring"):
        B.byz_distill_loss(torch.zeros(1, 8).expand(2, 8), torch.zeros(2, 3), i)
    w = torch.zeros(8, 4, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="neighbouring"):
        B.byz_gated_ffn(w, w.t(), w.t())


def test_binding_refuses_shapes_and_types_that_do_not_belong_together():
    i = torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(ValueError, match="rows"):
        B.byz_distill_loss(torch.zeros(3, 8), torch.zeros(2, 3), i)
    with pytest.raises(ValueError, match="shape"):
        B.byz_distill_loss(torch.zeros(2, 8), torch.zeros(2, 4), i)
    with pytest.raises(ValueError, match="dtype"):
        B.byz_distill_loss(torch.zeros(2, 8), torch.zeros(2, 3), i.long())
    with pytest.raises(ValueError, match="dtype"):
        B.byz_distill_loss(torch.zeros(2, 8), torch.zeros(2, 3).half(), i)
    with pytest.raises(ValueError, match="pitch"):
        B.byz_distill_loss(torch.zeros(2, 8), torch.zeros(2, 5)[:, :3], i)
    w = torch.zeros(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="columns"):
        B.byz_gated_ffn(torch.zeros(4, 6, dtype=torch.bfloat16), w, w)
    with pytest.raises(ValueError, match="dtype"):
        B.byz_gated_ffn(torch.zeros(4, 8, dtype=torch.float16), w, w)
    with pytest.raises(ValueError, match="shape"):
        B.byz_gated_ffn(torch.zeros(4, 8, dtype=torch.bfloat16), w, w[:3])
    with pytest.raises(ValueError, match="pitch"):
        B.byz_gated_ffn(w, w, torch.zeros(4, 16, dtype=torch.bfloat16)[:, :8])
