"""CPU-side checks of include/gar_linear.h: every declared symbol is exported, the struct mirrors match, and wrong
arguments are refused before any CUDA call."""
import ctypes as C
import os
import re
import subprocess

import pytest

import __graft_entry__ as entry

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, WORKSPACE = 1, 3, 4
BIG = 1 << 44                                                # a device buffer far from the others


@pytest.fixture(scope="module")
def pkg():
    entry.build()
    import paper_1905_04374_b200 as p
    return p


def test_every_declared_symbol_is_exported(pkg):
    text = open(os.path.join(ROOT, "include", "gar_linear.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(gar_[a-z_0-9]+)\s*\(", text)))
    assert len(names) == 9
    for name in names:
        assert hasattr(pkg.lib(), name), f"{name} declared in gar_linear.h but not exported"
        assert hasattr(pkg, name), f"{name} has no Python entry point"


def test_struct_mirrors_match_the_header(pkg, tmp_path):
    mirrors = {"gar_linear_logprobs_params_t": pkg.GarLinearLogprobsParams, "gar_linear_logprobs_grad_params_t": pkg.GarLinearLogprobsGradParams,
               "gar_gated_linear_params_t": pkg.GarGatedLinearParams, "gar_gated_linear_grad_params_t": pkg.GarGatedLinearGradParams,
               "gar_dropout_params_t": pkg.GarDropoutParams}
    lines, want = [], []
    for name, cls in mirrors.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(cls))
        for field, _ in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {field}));')
            want.append(getattr(cls, field).offset)
    src = tmp_path / "sz.cpp"
    src.write_text('#include "gar_linear.h"\n#include <cstdio>\n#include <cstddef>\nint main(){' + "".join(lines) + "}")
    exe = tmp_path / "sz"
    subprocess.check_call(["g++", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    assert [int(v) for v in subprocess.check_output([str(exe)]).split()] == want


def refuses(pkg, call, params, cases, status=INVALID):
    """Every change to the valid parameters is refused with `status`."""
    fn = getattr(pkg.linear.lib(), call)
    for change in cases:
        p = params()
        for key, value in change.items():
            *path, last = key.split(".")
            obj = p
            for part in path:
                obj = getattr(obj, part)
            setattr(obj, last, value)
        assert fn(C.byref(p)) == status, change
    assert fn(None) == INVALID


def sizes(pkg, call, params):
    return getattr(pkg.linear.lib(), call)(C.byref(params))


def saved(pkg, q, scales, ldq):
    s = pkg.GarCheckpoint()
    s.q, s.scales, s.ldq = q, scales, ldq
    return s


def test_scores_refusals(pkg):
    def params():
        p = pkg.GarLinearLogprobsParams()
        p.dtype, p.rows, p.hidden, p.vocab, p.ldx = 1, 4, 64, 100, 72
        p.x, p.weight, p.bias, p.targets, p.logprobs, p.lse, p.lse_lo = (1 << b for b in range(20, 27))
        p.workspace, p.workspace_bytes = BIG, 1 << 20
        return p
    call = "gar_linear_logprobs"
    refuses(pkg, call, params, [
        dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(hidden=0), dict(vocab=0), dict(ldx=63), dict(ldw=10), dict(x=None), dict(weight=None),
        dict(x=(1 << 20) + 1), dict(weight=(1 << 21) + 1), dict(bias=(1 << 22) + 1), dict(targets=None), dict(logprobs=None, lse=None, lse_lo=None),
        dict(lse=(1 << 20) + 64), dict(logprobs=1 << 21), dict(lse=(1 << 24) + 8), dict(lse_lo=1 << 22), dict(workspace=1 << 20), dict(rows=1 << 60)])
    refuses(pkg, call, params, [dict(dtype=0), dict(vocab=1 << 31), dict(hidden=1 << 31, ldx=0), dict(rows=1 << 30)], UNSUPPORTED)
    need = sizes(pkg, 'gar_linear_logprobs_workspace_bytes', params())
    assert need == 4 * 512 * 8 + 256                         # the parts of few rows, the targets' logits; x and W lie on 16 bytes
    refuses(pkg, call, params, [dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=BIG + 128)], WORKSPACE)
    p = params()
    p.ldx = 65
    assert sizes(pkg, 'gar_linear_logprobs_workspace_bytes', p) == need + 4 * 64 * 2
    p = params()
    p.rows = 0                                               # nothing to do: accepted without a GPU
    assert pkg.linear.lib().gar_linear_logprobs(C.byref(p)) == 0
    assert pkg.linear.lib().gar_linear_logprobs_workspace_bytes(None) == 0


def test_vectors_off_their_alignment_are_refused(pkg):
    def scores():
        p = pkg.GarLinearLogprobsParams()
        p.dtype, p.rows, p.hidden, p.vocab = 1, 4, 64, 100
        p.x, p.weight, p.bias, p.targets, p.logprobs, p.lse, p.lse_lo = (1 << b for b in range(20, 27))
        p.workspace, p.workspace_bytes = BIG, 1 << 20
        return p

    def grads():
        p = pkg.GarLinearLogprobsGradParams()
        p.dtype, p.workers, p.tokens, p.hidden, p.vocab = 1, 1, 4, 64, 100
        p.x, p.weight, p.bias, p.targets, p.lse, p.lse_lo, p.grad_logprobs, p.dx = (1 << b for b in range(20, 28))
        p.workspace, p.workspace_bytes = BIG, 1 << 24
        return p
    refuses(pkg, "gar_linear_logprobs", scores, [dict(targets=(1 << 23) + 4), dict(logprobs=(1 << 24) + 2), dict(lse=(1 << 25) + 2), dict(lse_lo=(1 << 26) + 1)])
    refuses(pkg, "gar_linear_logprobs_backward", grads, [dict(targets=(1 << 23) + 4), dict(lse=(1 << 24) + 2), dict(lse_lo=(1 << 25) + 1),
                                                         dict(grad_logprobs=(1 << 26) + 2)])


def test_scores_backward_refusals(pkg):
    def params():
        p = pkg.GarLinearLogprobsGradParams()
        p.dtype, p.grads_dtype, p.workers, p.tokens, p.hidden, p.vocab = 2, 0, 3, 4, 64, 100
        p.x, p.weight, p.bias, p.targets, p.lse, p.lse_lo, p.grad_logprobs, p.dx, p.weight_grads = (1 << b for b in range(20, 29))
        p.bias_grads, p.ld_grads = (1 << 28) + 4 * 6400, 6500
        p.workspace, p.workspace_bytes = BIG, 1 << 24
        return p
    call = "gar_linear_logprobs_backward"
    refuses(pkg, call, params, [
        dict(dtype=3), dict(grads_dtype=3), dict(workers=0), dict(tokens=-1), dict(hidden=0), dict(vocab=0), dict(ldx=63), dict(ldw=63), dict(lddx=63),
        dict(x=None), dict(weight=None), dict(targets=None), dict(lse=None), dict(grad_logprobs=None), dict(dx=None, weight_grads=None, bias_grads=None),
        dict(weight_grads=None), dict(ld_grads=6399), dict(ld_grads=-1), dict(ld_grads=1 << 60), dict(weight_grads=(1 << 28) + 2),
        dict(bias_grads=(1 << 28) + 4 * 6399), dict(dx=1 << 20), dict(dx=(1 << 20) + 64), dict(dx=1 << 21), dict(weight_grads=1 << 26, bias_grads=None),
        dict(x=(1 << 20) + 1), dict(dx=(1 << 27) + 1), dict(bias=(1 << 22) + 1), dict(workspace=1 << 27)])
    refuses(pkg, call, params, [dict(dtype=0), dict(workers=65, ld_grads=0), dict(tokens=1 << 30), dict(vocab=1 << 31), dict(hidden=1 << 31)], UNSUPPORTED)
    need = sizes(pkg, 'gar_linear_logprobs_backward_workspace_bytes', params())
    assert need > 0
    refuses(pkg, call, params, [dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=BIG + 16)], WORKSPACE)
    p = params()
    p.tokens, p.weight_grads, p.bias_grads = 0, None, None
    assert pkg.linear.lib().gar_linear_logprobs_backward(C.byref(p)) == 0


@pytest.mark.parametrize("tokens,vocab", [(1, 1), (300, 1000), (2048, 131072), (100000, 131072), (1 << 20, 50001)])
def test_gradient_is_kept_in_pieces(pkg, tokens, vocab):
    """The workspace holds 96 MB of the logits' gradient at most (256 columns of it, where the rows are that many), not rows x vocab of it."""
    p = pkg.GarLinearLogprobsGradParams()
    p.dtype, p.grads_dtype, p.workers, p.tokens, p.hidden, p.vocab = 1, 1, 1, tokens, 64, vocab
    p.x, p.weight, p.targets, p.lse, p.grad_logprobs, p.weight_grads = 1 << 40, 1 << 41, 1 << 42, 1 << 43, 1 << 44, 1 << 45
    rest = tokens * (64 * 2 + 4) + (1 << 22)
    assert 0 < sizes(pkg, 'gar_linear_logprobs_backward_workspace_bytes', p) <= max(96 << 20, tokens * 512) + rest


def test_gated_refusals(pkg):
    def params():
        p = pkg.GarGatedLinearParams()
        p.dtype, p.act, p.group, p.rows, p.hidden, p.inner = 1, 2, 64, 8, 64, 104
        p.x, p.w_gate, p.w_up, p.b_gate, p.b_up, p.y = (1 << b for b in range(20, 26))
        p.gate_saved, p.up_saved, p.y_saved = (saved(pkg, 1 << b, 1 << (b + 1), 112) for b in (27, 29, 31))
        return p
    call = "gar_gated_linear_forward"
    refuses(pkg, call, params, [
        dict(dtype=3), dict(act=4), dict(act=-1), dict(group=16), dict(rows=-1), dict(hidden=0), dict(inner=0), dict(ldx=63), dict(ld_gate=63),
        dict(ld_up=63), dict(ldy=99), dict(x=None), dict(w_gate=None), dict(w_up=None), dict(y=None), dict(x=(1 << 20) + 1), dict(b_up=(1 << 24) + 1),
        {"gate_saved.ldq": 96}, {"up_saved.ldq": 120}, {"y_saved.q": (1 << 31) + 8}, {"gate_saved.scales": None}, dict(y=1 << 20), dict(y=1 << 21),
        dict(y=(1 << 23) - 2), {"up_saved.q": 1 << 20}, {"y_saved.scales": 1 << 28}])
    refuses(pkg, call, params, [dict(dtype=0), dict(inner=1 << 31, **{"gate_saved.q": None, "up_saved.q": None, "y_saved.q": None})], UNSUPPORTED)
    assert sizes(pkg, 'gar_gated_linear_workspace_bytes', params()) == 0
    refuses(pkg, call, params, [dict(ldx=65), dict(w_up=(1 << 22) + 2), dict(ldx=65, workspace=BIG, workspace_bytes=100)], WORKSPACE)
    p = params()
    p.rows = 0
    assert pkg.linear.lib().gar_gated_linear_forward(C.byref(p)) == 0

    def grads():
        p = pkg.GarGatedLinearGradParams()
        p.dtype, p.act, p.group, p.rows, p.hidden, p.inner = 1, 2, 64, 8, 64, 104
        p.dy, p.w_gate, p.w_up, p.dgate, p.dup, p.dx = (1 << b for b in range(20, 26))
        p.gate_saved, p.up_saved = saved(pkg, 1 << 27, 1 << 28, 112), saved(pkg, 1 << 29, 1 << 30, 112)
        return p
    call = "gar_gated_linear_backward"
    refuses(pkg, call, grads, [
        dict(dtype=5), dict(act=7), dict(group=8), dict(dy=None), dict(w_gate=None), dict(dgate=None), dict(dup=None), dict(lddy=99), dict(ld_dgate=99),
        dict(ld_dup=99), dict(lddx=63), {"gate_saved.q": None}, {"up_saved.q": None}, {"up_saved.ldq": 100}, dict(dup=1 << 20), dict(dup=1 << 23),
        dict(dgate=(1 << 20) + 16), dict(dx=1 << 20), dict(dx=1 << 21), dict(dx=1 << 27), dict(dx=(1 << 25) + 1)])
    refuses(pkg, call, grads, [dict(dtype=0)], UNSUPPORTED)
    refuses(pkg, call, grads, [dict(ld_gate=65)], WORKSPACE)
    p = grads()
    p.rows, p.dgate = 0, 1 << 20                             # in place
    assert pkg.linear.lib().gar_gated_linear_backward(C.byref(p)) == 0


def test_dropout_refusals(pkg):
    def params():
        p = pkg.GarDropoutParams()
        p.dtype, p.p, p.rows, p.cols, p.ldx = 0, 0.5, 8, 100, 104
        p.x, p.residual, p.y, p.counter = 1 << 20, 1 << 21, 1 << 22, 1 << 23
        return p
    call = "gar_dropout"
    refuses(pkg, call, params, [
        dict(dtype=3), dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(rows=-1), dict(cols=0), dict(ldx=99), dict(ldy=99), dict(ld_residual=99),
        dict(x=None), dict(y=None), dict(x=(1 << 20) + 2), dict(counter=(1 << 23) + 4), dict(y=1 << 20), dict(y=(1 << 21) + 4), dict(y=(1 << 23) - 40)])
    refuses(pkg, call, params, [dict(cols=1 << 32, ldx=0)], UNSUPPORTED)
    p = params()
    p.rows, p.y, p.ldy = 0, 1 << 20, 104                     # in place
    assert pkg.linear.lib().gar_dropout(C.byref(p)) == 0
