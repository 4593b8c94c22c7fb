"""CPU-side checks of include/gar_worker.h: every declared symbol is exported, the struct mirrors
match, and wrong arguments are refused before any CUDA call (this machine needs no GPU for that)."""
import ctypes as C
import os
import re
import subprocess

import pytest

import __graft_entry__ as entry

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED = 1, 3


@pytest.fixture(scope="module")
def pkg():
    entry.build()
    import paper_1905_04374_b200 as p
    return p


def test_every_declared_symbol_is_exported(pkg):
    text = open(os.path.join(ROOT, "include", "gar_worker.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = sorted(set(re.findall(r"\b(gar_[a-z_0-9]+)\s*\(", text)))
    assert len(names) == 9
    for name in names:
        assert hasattr(pkg.lib(), name), f"{name} declared in gar_worker.h but not exported"
        # the question whether to bring a workspace is asked inside the binding
        assert hasattr(pkg, name) or name == "gar_weight_grad_wants_workspace", f"{name} has no Python entry point"


def test_struct_mirrors_match_the_header(pkg, tmp_path):
    mirrors = {"gar_checkpoint_t": pkg.GarCheckpoint, "gar_logprobs_params_t": pkg.GarLogprobsParams,
               "gar_logprobs_grad_params_t": pkg.GarLogprobsGradParams, "gar_activation_params_t": pkg.GarActivationParams,
               "gar_activation_grad_params_t": pkg.GarActivationGradParams, "gar_weight_grad_params_t": pkg.GarWeightGradParams}
    lines, want = [], []
    for name, cls in mirrors.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(cls))
        for field, _ in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {field}));')
            want.append(getattr(cls, field).offset)
    src = tmp_path / "sz.cpp"
    src.write_text('#include "gar_worker.h"\n#include <cstdio>\n#include <cstddef>\nint main(){' + "".join(lines) + "}")
    exe = tmp_path / "sz"
    subprocess.check_call(["g++", "-I" + os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    assert [int(v) for v in subprocess.check_output([str(exe)]).split()] == want


def refuses(pkg, call, params, cases, status=INVALID):
    """Every change to the valid parameters is refused with `status`."""
    fn = getattr(pkg.worker.lib(), call)
    for change in cases:
        p = params()
        for key, value in change.items():
            target, *path = key.split(".")
            obj = p
            for part in [target] + path[:-1] if path else []:
                obj = getattr(obj, part)
            setattr(obj, path[-1] if path else target, value)
        assert fn(C.byref(p)) == status, change
    assert fn(None) == INVALID


def test_logprobs_refusals(pkg):
    def params():
        p = pkg.GarLogprobsParams()
        p.dtype, p.rows, p.vocab, p.ld, p.top = 1, 4, 100, 104, 2
        p.logits, p.targets, p.logprobs, p.entropy, p.lse = 1 << 20, 1 << 21, 1 << 22, 1 << 23, 1 << 24
        p.top_logprobs, p.top_index = 1 << 25, 1 << 26
        return p
    refuses(pkg, "gar_token_logprobs", params, [
        dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(vocab=0), dict(ld=99), dict(logits=None), dict(logits=(1 << 20) + 1),
        dict(top=-1), dict(top=33), dict(vocab=1, ld=0), dict(targets=None), dict(top=0), dict(top_logprobs=None),
        dict(top_index=None), dict(lse=(1 << 20) + 64), dict(entropy=(1 << 22) + 8), dict(rows=1 << 60),
        dict(logprobs=None, entropy=None, lse=None, top=0, top_logprobs=None, top_index=None)])
    refuses(pkg, "gar_token_logprobs", params, [dict(vocab=1 << 31, ld=0)], UNSUPPORTED)
    p = params()
    p.rows = 0                                               # nothing to do: accepted without a GPU
    assert pkg.worker.lib().gar_token_logprobs(C.byref(p)) == 0


def test_logprobs_backward_refusals(pkg):
    def params():
        p = pkg.GarLogprobsGradParams()
        p.dtype, p.rows, p.vocab, p.top = 0, 4, 100, 2
        p.logits, p.targets, p.lse, p.entropy, p.top_index = 1 << 20, 1 << 21, 1 << 22, 1 << 23, 1 << 24
        p.grad_logprobs, p.grad_entropy, p.grad_top, p.dlogits = 1 << 25, 1 << 26, 1 << 27, 1 << 28
        return p
    refuses(pkg, "gar_token_logprobs_backward", params, [
        dict(dtype=5), dict(ld=99), dict(ld_dlogits=99), dict(dlogits=None), dict(lse=None), dict(logits=None), dict(targets=None),
        dict(entropy=None), dict(top_index=None), dict(grad_top=None), dict(top=0), dict(top=40), dict(dlogits=(1 << 28) + 2),
        dict(dlogits=(1 << 20) + 16), dict(dlogits=1 << 20, ld_dlogits=200), dict(dlogits=1 << 25)])
    refuses(pkg, "gar_token_logprobs_backward", params, [dict(vocab=1 << 31)], UNSUPPORTED)
    p = params()
    p.rows, p.dlogits = 0, 1 << 20                           # in place
    assert pkg.worker.lib().gar_token_logprobs_backward(C.byref(p)) == 0


def _saved(pkg, q, scales, ldq):
    s = pkg.GarCheckpoint()
    s.q, s.scales, s.ldq = q, scales, ldq
    return s


def test_activation_refusals(pkg):
    def params():
        p = pkg.GarActivationParams()
        p.dtype, p.act, p.group, p.rows, p.cols = 1, 2, 64, 8, 100
        p.x, p.up, p.y = 1 << 20, 1 << 21, 1 << 22
        p.x_saved, p.up_saved, p.y_saved = (_saved(pkg, 1 << b, 1 << (b + 1), 112) for b in (23, 25, 27))
        return p
    refuses(pkg, "gar_activation_forward", params, [
        dict(dtype=3), dict(act=4), dict(act=-1), dict(group=16), dict(group=0), dict(cols=0), dict(rows=-1), dict(ldx=50),
        dict(ldup=50), dict(ldy=50), dict(x=None), dict(x=(1 << 20) + 1), {"x_saved.ldq": 96}, {"x_saved.ldq": 120},
        {"x_saved.q": (1 << 23) + 8}, {"y_saved.scales": None}, dict(up=None), dict(y=(1 << 20) + 32), dict(y=1 << 21),
        {"y_saved.q": 1 << 23}, {"x_saved.q": 1 << 20}, {"x_saved.scales": (1 << 25) + 4}])

    def none(p=params):
        q = p()
        q.up, q.y = None, None
        for s in (q.x_saved, q.up_saved, q.y_saved):
            s.q = None
        return q
    refuses(pkg, "gar_activation_forward", none, [dict()])   # nothing to write

    def grads():
        p = pkg.GarActivationGradParams()
        p.dtype, p.act, p.group, p.rows, p.cols = 2, 3, 32, 8, 100
        p.dy, p.dx, p.dup = 1 << 20, 1 << 21, 1 << 22
        p.x_saved, p.up_saved = _saved(pkg, 1 << 23, 1 << 24, 112), _saved(pkg, 1 << 25, 1 << 26, 112)
        return p
    refuses(pkg, "gar_activation_backward", grads, [
        dict(dtype=-2), dict(act=9), dict(group=256), dict(dy=None), dict(dx=None), dict(dup=None), {"up_saved.q": None},
        {"x_saved.q": None}, {"x_saved.scales": None}, {"up_saved.ldq": 100}, dict(lddx=99), dict(lddup=99), dict(dup=1 << 21),
        dict(dup=1 << 20), dict(dx=(1 << 20) + 2), dict(dx=1 << 23)])
    # column ranges of one wider buffer are no overlap
    p = grads()
    p.rows = 0
    assert pkg.worker.lib().gar_activation_backward(C.byref(p)) == 0
    L = pkg.worker.lib()
    s = _saved(pkg, 1 << 23, 1 << 24, 112)
    assert L.gar_checkpoint_pack(1, 1 << 20, 8, 100, 0, 48, C.byref(s), None) == INVALID
    assert L.gar_checkpoint_pack(1, 1 << 20, 8, 100, 0, 64, None, None) == INVALID
    assert L.gar_checkpoint_unpack(1, C.byref(s), 8, 100, 64, None, 0, None) == INVALID
    assert L.gar_checkpoint_unpack(1, C.byref(s), 8, 100, 64, 1 << 23, 0, None) == INVALID
    assert L.gar_checkpoint_unpack(1, C.byref(s), 0, 100, 64, 1 << 20, 0, None) == 0


def test_weight_grad_refusals(pkg):
    def params():
        p = pkg.GarWeightGradParams()
        p.dtype, p.grads_dtype, p.group, p.workers, p.tokens, p.out_features, p.in_features = 1, 0, 128, 3, 10, 20, 30
        p.dy, p.lengths, p.weight_grads, p.bias_grads, p.ld_grads = 1 << 20, 1 << 21, 1 << 22, (1 << 22) + 4 * 600, 620
        p.x_saved = _saved(pkg, 1 << 23, 1 << 24, 32)
        return p
    refuses(pkg, "gar_linear_weight_grad", params, [
        dict(dtype=7), dict(grads_dtype=3), dict(group=100), dict(workers=0), dict(tokens=-1), dict(out_features=0), dict(in_features=0),
        dict(dy=None), dict(weight_grads=None), dict(ld_dy=19), dict(ld_grads=599), dict(ld_grads=-1), {"x_saved.q": None},
        {"x_saved.ldq": 16}, dict(bias_grads=(1 << 22) + 4 * 599), dict(bias_grads=(1 << 22) + 4 * 601), dict(dy=1 << 22),
        dict(weight_grads=(1 << 22) + 2), dict(lengths=1 << 22), dict(ld_grads=1 << 60)])
    L = pkg.worker.lib()
    need = L.gar_weight_grad_workspace_bytes(C.byref(params()))
    assert need == 30 * 32 * 2 + 256 - (30 * 32 * 2) % 256 + 30 * 24 * 2 + 256 - (30 * 24 * 2) % 256      # x, and dy (rows of 20)
    refuses(pkg, "gar_linear_weight_grad", params, [
        dict(workspace=1 << 30, workspace_bytes=need - 1), dict(workspace=(1 << 30) + 128, workspace_bytes=need)], 4)
    refuses(pkg, "gar_linear_weight_grad", params, [dict(workspace=1 << 20, workspace_bytes=need)])
    refuses(pkg, "gar_linear_weight_grad", params, [
        dict(dtype=0), dict(workers=65, ld_grads=1 << 40), dict(out_features=1 << 31), dict(tokens=1 << 30)], UNSUPPORTED)


@pytest.mark.parametrize("change,cut", [(dict(), False), (dict(tokens=512), False), (dict(tokens=513), True), (dict(lengths=1 << 21), True),
                                        (dict(dy=(1 << 20) + 2), True), (dict(out_features=256), True)])
def test_weight_grad_panels_are_not_cut(pkg, change, cut):
    """Up to 512 tokens without lengths, more than 256 outputs, aligned dy: panels, whose tokens stay whole however
    few the output tiles are; otherwise these few tiles are cut into parts, which need a workspace."""
    p = pkg.GarWeightGradParams()
    p.dtype, p.grads_dtype, p.group, p.workers, p.tokens, p.out_features, p.in_features = 1, 0, 64, 5, 473, 616, 15
    p.dy, p.weight_grads, p.ld_grads, p.x_saved = 1 << 20, 1 << 28, 616 * 15, _saved(pkg, 1 << 23, 1 << 24, 16)
    for name, value in change.items():
        setattr(p, name, value)
    L = pkg.worker.lib()
    assert (L.gar_weight_grad_wants_workspace(C.byref(p)) != 0) == cut
    assert (L.gar_weight_grad_workspace_bytes(C.byref(p)) > 0) == cut
