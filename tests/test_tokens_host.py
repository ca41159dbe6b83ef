"""The token operators through the C-ABI and the binding, without a GPU: constants and the form's layout, the
generator's published answers, and what a kernel could not take is refused before any launch."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2010_04902_amd as B
from paper_2010_04902_amd import worker_tokens as W
from token_forms import philox

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, ENOMEM = 0, -1, -3
P = 0x10000  # an address nothing reads: every call below returns before a launch
NAN, INF = float("nan"), float("inf")


def test_header_agrees_with_the_binding(tmp_path):
    src = tmp_path / "consts.c"
    fields = [name for name, _ in B.byz_residual_form._fields_]
    names = ["offset_at" if name == "_offset_at" else name for name in fields]
    src.write_text('''#include <stddef.h>
#include <stdio.h>
#include "byzshield_worker.h"
int main(void) {
    printf("%%d %%d %%d %%zu", BYZ_NORM_NONE, BYZ_NORM_RMS, BYZ_NORM_LAYER, sizeof(byz_residual_form));
%s
    return 0;
}
''' % "\n".join('    printf(" %%zu", offsetof(byz_residual_form, %s));' % name for name in names))
    exe = tmp_path / "consts"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)],
                   check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [B.BYZ_NORM_NONE, B.BYZ_NORM_RMS, B.BYZ_NORM_LAYER, ctypes.sizeof(B.byz_residual_form)] + [
        getattr(B.byz_residual_form, name).offset for name in fields]


def test_generator_gives_its_published_answers():
    answers = [((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
               ((2 ** 32 - 1,) * 4, (2 ** 32 - 1,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
               ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
                (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))]
    for counter, key, want in answers:
        assert tuple(int(w[()]) for w in philox([np.uint64(c) for c in counter], key)) == want


def test_form_keeps_any_64_bits():
    form = B.byz_residual_form(seed=-1, offset=2 ** 64 + 5)
    assert form.seed == 2 ** 64 - 1 and form.offset == 5 and form.offset_at is None


# ------------------------------------------------------------------ C-ABI refusals


def _dropout(x=P, rows=4, cols=10, ld=10, dtype=0, p=0.1, seed=1, offset=2, at=None, first=0, y=P, y_ld=10):
    return W._load().byz_dropout(x, rows, cols, ld, dtype, p, seed, offset, at, first, y, y_ld, None)


@pytest.mark.parametrize("bad", [
    dict(x=None), dict(y=None), dict(rows=-1), dict(cols=-1), dict(cols=2 ** 31, ld=2 ** 31, y_ld=2 ** 31), dict(ld=9), dict(y_ld=9),
    dict(dtype=3), dict(dtype=-1), dict(p=-0.1), dict(p=1.5), dict(p=NAN), dict(at=P + 4), dict(first=-1), dict(first=2 ** 32 - 3),
    dict(rows=2 ** 32 + 1), dict(x=P + 2), dict(y=P + 1), dict(ld=1 << 62), dict(y_ld=1 << 62)], ids=str)
def test_dropout_refusals(bad):
    assert _dropout(**bad) == EINVAL


def test_dropout_of_nothing():
    assert _dropout(rows=0, x=None, y=None) == OK and _dropout(cols=0) == OK


FORM = dict(post=1, pre=1)


def _residual(x=P, x_ld=10, h=P, h_ld=10, rows=4, cols=10, dtype=0, form=FORM, w1=None, b1=None, gate=None, gate_rows=4, w2=None,
              b2=None, out=P, out_ld=10, y=P, y_ld=10, stats=P):
    f = None if form is None else B.byz_residual_form(**form)
    return W._load().byz_residual_norm(x, x_ld, h, h_ld, rows, cols, dtype, f, w1, b1, gate, gate_rows, w2, b2, out, out_ld, y, y_ld,
                                       stats, None)


SHARED = [
    dict(x=None), dict(rows=-1), dict(cols=0), dict(cols=-4), dict(cols=2 ** 31), dict(dtype=3), dict(x_ld=9), dict(h_ld=9),
    dict(x=P + 2), dict(h=P + 1), dict(form=None), dict(form=dict(post=3)), dict(form=dict(pre=-1)), dict(form=dict(eps=-1.0)),
    dict(form=dict(eps=NAN)), dict(form=dict(scale=INF)), dict(form=dict(scale=NAN)), dict(form=dict(p=1.01)),
    dict(form=dict(first_row=-1)), dict(form=dict(first_row=2 ** 32)), dict(w1=P + 2), dict(gate=P, gate_rows=0),
    dict(gate=P, gate_rows=-2), dict(gate=P + 1), dict(w2=P + 3), dict(rows=2 ** 33), dict(x_ld=1 << 62),
    dict(h=None), dict(h=None, form=dict(post=0, pre=1), gate=P), dict(h=None, form=dict(post=0, pre=0)),
    dict(form=dict(post=1, pre=0), w2=P)]


@pytest.mark.parametrize("bad", SHARED + [
    dict(out=None), dict(y=None), dict(out_ld=9), dict(y_ld=9), dict(out=P + 2), dict(y=P + 1), dict(stats=P + 2), dict(b1=P + 1),
    dict(b2=P + 1), dict(form=dict(post=1, pre=0), b2=P)], ids=str)
def test_residual_refusals(bad):
    assert _residual(**bad) == EINVAL


def test_residual_of_nothing():
    assert _residual(rows=0, x=None, h=None, out=None, y=None) == OK


def _residual_backward(dout=P, dout_ld=10, dy=P, dy_ld=10, x=P, x_ld=10, h=P, h_ld=10, stats=P, rows=4, cols=10, dtype=0, form=FORM,
                       w1=None, b1=None, gate=None, gate_rows=4, w2=None, dx=P, dx_ld=10, dh=P, dh_ld=10, dw1=None, db1=None,
                       dgate=None, dw2=None, db2=None, ws=P, nbytes=1 << 30):
    f = None if form is None else B.byz_residual_form(**form)
    return W._load().byz_residual_norm_backward(dout, dout_ld, dy, dy_ld, x, x_ld, h, h_ld, stats, rows, cols, dtype, f, w1, b1, gate,
                                                gate_rows, w2, dx, dx_ld, dh, dh_ld, dw1, db1, dgate, dw2, db2, ws, nbytes, None)


@pytest.mark.parametrize("bad", SHARED + [
    dict(dout=None, dy=None), dict(dx=None), dict(dh=None), dict(stats=None), dict(stats=P + 2), dict(dout_ld=9), dict(dy_ld=3),
    dict(dx_ld=9), dict(dh_ld=9), dict(dout=P + 2), dict(dy=P + 1), dict(dx=P + 2), dict(dh=P + 2), dict(dgate=P), dict(dw1=P + 2),
    dict(db1=P + 1), dict(dw2=P + 1), dict(db2=P + 1), dict(gate=P, dgate=P + 2), dict(form=dict(post=1, pre=0)),
    dict(form=dict(post=1, pre=0), dy=None, dw2=P), dict(form=dict(post=0, pre=1), h=None, dw1=P)], ids=str)
def test_residual_backward_refusals(bad):
    assert _residual_backward(**bad) == EINVAL


def test_residual_backward_needs_its_workspace():
    need = W._load().byz_residual_norm_backward_workspace_bytes(4, 10, 0, 4)
    assert need > 0
    for bad in (dict(ws=None), dict(ws=P + 4), dict(nbytes=need - 1)):
        assert _residual_backward(**bad) == ENOMEM
    for sizes in ((-1, 10, 0, 4), (4, 0, 0, 4), (4, 10, 9, 4), (4, 10, 0, 0), (1 << 40, 1 << 30, 0, 1)):
        assert W._load().byz_residual_norm_backward_workspace_bytes(*sizes) == 0


ROWS = dict(logits=P, rows=4, vocab=100, ld=100, dtype=0, label=P)
WORK = dict(ws=P, nbytes=1 << 20)
GRADIENT = dict(dlogits=P, dld=100)
POLICY = dict(old=P, advantage=P, ref=P, clip_low=0.2, clip_high=0.2, kl=0.1, temperature=1.0)
PAIRS = dict(bounds=P, pairs=2)
CALLS = {
    "byz_token_logp": {**ROWS, "temperature": 1.0, "logp": P, "stats": P, **WORK},
    "byz_token_logp_backward": {"dloss": P, **ROWS, "stats": P, "temperature": 1.0, **GRADIENT, **WORK},
    "byz_policy_loss": {**ROWS, **POLICY, "loss": P, "logp": P, "stats": P, **WORK},
    "byz_policy_loss_backward": {"dloss": P, **ROWS, **POLICY, "stats": P, **GRADIENT, **WORK},
    "byz_policy_loss_step": {"dloss": P, **ROWS, **POLICY, "loss": P, "logp": P, **GRADIENT, **WORK},
    "byz_preference_loss": {**ROWS, **PAIRS, "ref": P, "beta": 0.1, "smoothing": 0.0, "temperature": 1.0, "loss": P, "sums": P,
                            "slope": P, "stats": P, **WORK},
    "byz_preference_loss_backward": {"dloss": P, **ROWS, **PAIRS, "slope": P, "beta": 0.1, "temperature": 1.0, "stats": P, **GRADIENT,
                                     **WORK},
    "byz_preference_loss_step": {"dloss": P, **ROWS, **PAIRS, "ref": P, "beta": 0.1, "smoothing": 0.0, "temperature": 1.0, "loss": P,
                                 "sums": P, **GRADIENT, **WORK},
}
WRONG = {
    "logits": [None, P + 2], "rows": [-1, 1 << 40], "vocab": [0, -5, 1 << 31], "ld": [99, 1 << 62], "dtype": [-1, 3],
    "label": [None, P + 2], "temperature": [0.0, -1.0, NAN, INF], "dloss": [None, P + 1], "dlogits": [None, P + 2],
    "dld": [99, 1 << 62], "old": [None, P + 2], "advantage": [None, P + 2], "clip_low": [-0.1, 1.1, NAN],
    "clip_high": [-0.1, NAN, INF], "kl": [-1.0, NAN, INF], "bounds": [None, P + 2], "pairs": [-1, 1 << 40], "beta": [NAN, INF],
    "smoothing": [-0.1, 1.1, NAN], "stats": [P + 2], "logp": [P + 2], "loss": [None, P + 2], "sums": [P + 2], "slope": [P + 2], "ref": [P + 2],
}


@pytest.mark.parametrize("name", CALLS)
def test_loss_refusals(name):
    call = getattr(W._load(), name)
    for argument, values in WRONG.items():
        if argument in CALLS[name]:
            for value in values:
                got = call(*{**CALLS[name], argument: value}.values(), None)
                assert got == EINVAL, (argument, value)
    if name.endswith("_backward"):
        assert call(*{**CALLS[name], "stats": None}.values(), None) == EINVAL
    if name == "byz_token_logp":
        assert call(*{**CALLS[name], "logp": None}.values(), None) == EINVAL
    if "policy" in name:
        assert call(*{**CALLS[name], "ref": None}.values(), None) == EINVAL  # kl is not 0
    if name == "byz_preference_loss_backward":
        assert call(*{**CALLS[name], "slope": None}.values(), None) == EINVAL
    need = W._load().byz_token_loss_workspace_bytes(4, 100, 0)
    assert need > 0
    for bad in (dict(ws=None), dict(ws=P + 8), dict(nbytes=need - 1)):
        assert call(*{**CALLS[name], **bad}.values(), None) == ENOMEM


@pytest.mark.parametrize("name", CALLS)
def test_losses_refuse_temperatures_next_to_0(name):
    for value in (2.0 ** -65, 1e-30, 2.0 ** -149):
        assert getattr(W._load(), name)(*{**CALLS[name], "temperature": value}.values(), None) == EINVAL


@pytest.mark.parametrize("name", CALLS)
def test_loss_without_rows(name):
    none = dict(rows=0, logits=None, label=None, ws=None, nbytes=0)
    if "preference" in name:
        none.update(pairs=0, bounds=None)
    assert getattr(W._load(), name)(*{**CALLS[name], **none}.values(), None) == OK


def test_loss_workspace_of_wrong_sizes():
    for sizes in ((-1, 10, 0), (4, 0, 0), (4, 1 << 31, 0), (4, 10, 5), (1 << 40, 10, 0)):
        assert W._load().byz_token_loss_workspace_bytes(*sizes) == 0


# ------------------------------------------------------------------ the binding's refusals


def test_binding_refuses_what_is_not_on_a_gpu():
    x, label = torch.zeros(4, 10), torch.zeros(4, dtype=torch.int32)
    rows, bounds = torch.zeros(4), torch.tensor([0, 2, 4], dtype=torch.int32)
    form = B.byz_residual_form()
    for call in (lambda: B.byz_dropout(x, 0.1, 1), lambda: B.byz_residual_norm(x, x, form),
                 lambda: B.byz_residual_norm_backward(x, x, x, x, torch.zeros(4, 4), form), lambda: B.byz_token_logp(x, label),
                 lambda: B.byz_token_logp_backward(rows, x, label, torch.zeros(4, 2)),
                 lambda: B.byz_policy_loss(x, label, rows, rows), lambda: B.byz_policy_loss_step(x, label, rows, rows, rows),
                 lambda: B.byz_policy_loss_backward(rows, x, label, rows, rows, torch.zeros(4, 2)),
                 lambda: B.byz_preference_loss(x, label, bounds), lambda: B.byz_preference_loss_step(x, label, bounds, rows[:1]),
                 lambda: B.byz_preference_loss_backward(rows[:1], x, label, bounds, rows[:1], torch.zeros(4, 2)),
                 lambda: B.byz_residual_form(offset_at=torch.zeros(1, dtype=torch.int64))):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_binding_refuses_other_layouts():
    for x in (torch.zeros(10), torch.zeros(2, 3, 4), torch.zeros(10, 4).t(), torch.zeros(4, 1).expand(4, 10)):
        with pytest.raises(ValueError):
            B.byz_dropout(x, 0.1, 1)


def test_binding_refuses_rows_that_would_wrap():
    for first_row in (2 ** 63, 2 ** 64, 2 ** 64 + 5, -2 ** 63 - 1):
        with pytest.raises(ValueError, match="first_row"):
            B.byz_residual_form(first_row=first_row)
        form = B.byz_residual_form(first_row=7)
        with pytest.raises(ValueError, match="first_row"):
            form.first_row = first_row
        assert form.first_row == 7
        with pytest.raises(ValueError, match="first_row"):
            B.byz_dropout(torch.zeros(4, 10), 0.1, 1, first_row=first_row)
