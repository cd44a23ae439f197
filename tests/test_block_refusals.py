"""What the calls of an experts block refuse: checked on the host before anything is launched, so no GPU is needed."""
import ctypes as C

import pytest

from paper_2307_00228_b200 import binding as B

P = 1 << 20   # addresses that are never followed: a refused call launches nothing


def _status(code, status):
    assert status == B.STATUS_NAMES.index(code), (B.STATUS_NAMES[status], B.it_last_error_message())


def norm(n=10, x=P, residual=None, sum_out=None, out=2 * P, scales=None, **kw):
    d = B.it_norm_desc(**{**dict(dim=64, feat_dtype=1, out_dtype=1, eps=1e-5, weight=None), **kw})
    return B.lib().it_residual_norm(C.byref(d), n, x, residual, sum_out, out, scales, None)


@pytest.mark.parametrize("kw", [dict(feat_dtype=2), dict(feat_dtype=7), dict(out_dtype=0), dict(dim=0), dict(dim=-8), dict(dim=12), dict(n=-1), dict(eps=-1.0),
                                dict(eps=float("nan")), dict(eps=float("inf")), dict(weight=P + 4), dict(x=None), dict(out=None), dict(x=P + 2), dict(out=2 * P + 8),
                                dict(residual=3 * P + 8), dict(sum_out=3 * P + 8), dict(out_dtype=2), dict(scales=3 * P), dict(out_dtype=2, dim=24, scales=3 * P),
                                dict(out=P + 16), dict(sum_out=P + 128), dict(sum_out=2 * P), dict(out_dtype=2, scales=3 * P, out=P), dict(out_dtype=2, scales=P),
                                dict(out_dtype=2, scales=2 * P), dict(residual=3 * P, sum_out=3 * P + 64), dict(weight=2 * P), dict(n=1 << 62)], ids=str)
def test_norm(kw):
    _status("IT_ERR_INVALID_ARG", norm(**kw))


def test_norm_null_description_and_no_rows():
    _status("IT_ERR_INVALID_ARG", B.lib().it_residual_norm(None, 1, P, None, None, 2 * P, None, None))
    _status("IT_OK", norm(n=0, x=None, out=None))


def route(n=10, logits=P, ids=2 * P, weights=3 * P, **kw):
    d = B.it_route_desc(**{**dict(n_experts=16, top_k=2, logit_dtype=0, score=0, balance_bias=None, n_groups=1, group_k=1, group_best=1, renormalise=1, weight_scale=1.0), **kw})
    return B.lib().it_route(C.byref(d), n, logits, ids, weights, None)


@pytest.mark.parametrize("kw", [dict(logit_dtype=2), dict(score=2), dict(score=-1), dict(n=-1), dict(n_experts=0), dict(top_k=0), dict(top_k=17), dict(n_groups=0), dict(n_groups=3),
                                dict(group_k=0), dict(group_k=2), dict(group_best=0), dict(group_best=3), dict(weight_scale=float("inf")), dict(weight_scale=float("nan")),
                                dict(logits=None), dict(ids=None), dict(weights=None), dict(logits=P + 2), dict(ids=2 * P + 1), dict(weights=3 * P + 2), dict(ids=P + 64),
                                dict(weights=P), dict(ids=3 * P), dict(balance_bias=2 * P), dict(balance_bias=P + 1), dict(n=1 << 61)], ids=str)
def test_route(kw):
    _status("IT_ERR_INVALID_ARG", route(**kw))


def test_route_limits():
    _status("IT_ERR_UNSUPPORTED", route(n_experts=1025))
    _status("IT_ERR_UNSUPPORTED", route(n_experts=64, top_k=33))
    _status("IT_ERR_INVALID_ARG", B.lib().it_route(None, 1, P, 2 * P, 3 * P, None))
    _status("IT_OK", route(n=0, logits=None, ids=None, weights=None))


BIG = 1 << 30


def experts(n=10, x=BIG, x_scale=None, ids=2 * BIG, weights=3 * BIG, out=4 * BIG, workspace=5 * BIG, bytes_=1 << 28, **kw):
    d = B.it_experts_desc(**{**dict(n_experts=4, top_k=2, in_dim=64, hidden_dim=128, out_dim=64, feat_dtype=1, in_dtype=1, act=1, gated=0, W1=6 * BIG, b1=None, W2=7 * BIG, b2=None,
                                    w1_scale=None), **kw})
    return B.lib().it_experts_forward(C.byref(d), n, x, x_scale, ids, weights, out, workspace, bytes_, None)


@pytest.mark.parametrize("kw", [dict(feat_dtype=2), dict(in_dtype=0), dict(act=4), dict(act=-1), dict(n=-1), dict(n_experts=0), dict(top_k=0), dict(in_dim=0), dict(hidden_dim=-8),
                                dict(out_dim=0), dict(in_dim=60), dict(hidden_dim=60), dict(out_dim=60), dict(hidden_dim=0, gated=1, W2=None), dict(W2=None), dict(hidden_dim=0),
                                dict(hidden_dim=0, W2=None, b2=8 * BIG), dict(W1=None), dict(x=None), dict(ids=None), dict(weights=None), dict(out=None), dict(x=BIG + 8),
                                dict(out=4 * BIG + 8), dict(W1=6 * BIG + 8), dict(W2=7 * BIG + 2), dict(b1=8 * BIG + 4), dict(b2=8 * BIG + 8), dict(ids=2 * BIG + 2),
                                dict(weights=3 * BIG + 1), dict(x_scale=9 * BIG), dict(w1_scale=9 * BIG), dict(in_dtype=2), dict(in_dtype=2, w1_scale=9 * BIG),
                                dict(in_dtype=2, in_dim=72, w1_scale=9 * BIG, x_scale=10 * BIG), dict(out=BIG), dict(out=2 * BIG), dict(out=5 * BIG), dict(x=5 * BIG + 4096),
                                dict(out=7 * BIG + 64), dict(W2=5 * BIG)], ids=str)
def test_experts(kw):
    _status("IT_ERR_INVALID_ARG", experts(**kw))


def test_experts_limits():
    _status("IT_ERR_UNSUPPORTED", experts(feat_dtype=0, in_dtype=2, w1_scale=9 * BIG, x_scale=10 * BIG))
    _status("IT_ERR_UNSUPPORTED", experts(n=1 << 31))
    _status("IT_ERR_UNSUPPORTED", experts(feat_dtype=0, in_dtype=0, n=400_000_000))
    _status("IT_ERR_UNSUPPORTED", experts(n_experts=1 << 24))
    _status("IT_ERR_WORKSPACE", experts(workspace=None))
    _status("IT_ERR_WORKSPACE", experts(workspace=5 * BIG + 64))
    _status("IT_ERR_WORKSPACE", experts(bytes_=300))
    _status("IT_ERR_INVALID_ARG", B.lib().it_experts_forward(None, 1, P, None, P, P, P, P, 0, None))
    _status("IT_ERR_INVALID_ARG", B.lib().it_experts_workspace_bytes(C.byref(B.it_experts_desc()), 1, None))
    _status("IT_ERR_WORKSPACE", B.lib().it_experts_check(None, None))


def test_layers_refuse_what_only_the_block_takes():
    """8-bit states and SiLU belong to the block: a layer with them is refused by its checks, as it was."""
    text = open(B.__file__.replace("binding.py", "csrc/api.cu")).read()
    assert "L->act <= IT_ACT_ELU" in text and "L->feat_dtype == IT_F32 || L->feat_dtype == IT_BF16" in text


def test_structures_match_the_header():
    import os
    import re
    import subprocess
    import tempfile
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    for s in (B.it_norm_desc, B.it_route_desc, B.it_experts_desc):
        fields = [f[0] for f in s._fields_]
        prog = "#include <stdio.h>\n#include <stddef.h>\n#include \"inferturbo.h\"\nint main(void){printf(\"%zu\", sizeof(" + s.__name__ + "));" + \
            "".join(f'printf(" %zu", offsetof({s.__name__}, {f}));' for f in fields) + "return 0;}\n"
        with tempfile.TemporaryDirectory() as d:
            src, exe = os.path.join(d, "t.c"), os.path.join(d, "t")
            open(src, "w").write(prog)
            subprocess.check_call(["gcc", "-I", os.path.join(root, "include"), src, "-o", exe])
            nums = [int(t) for t in subprocess.check_output([exe]).split()]
        assert nums == [C.sizeof(s)] + [getattr(s, f).offset for f in fields]
    assert re.search(r"IT_E4M3 = 2", open(os.path.join(root, "include", "inferturbo.h")).read())


def test_binding_refuses_tensors_that_the_library_could_not_tell():
    """Wrong types, shapes and places of tensors, which are addresses only to the library."""
    import torch
    with pytest.raises(ValueError, match="current CUDA device"):
        B.NormDesc(dim=8, feat_dtype=torch.float32, weight=torch.ones(8))
    with pytest.raises(ValueError, match="expected"):
        B.NormDesc(dim=8, feat_dtype=torch.float32, weight=torch.ones(9))
    with pytest.raises(TypeError):
        B.NormDesc(dim=8, feat_dtype=torch.float16)
    d = B.NormDesc(dim=8, feat_dtype=torch.float32)
    with pytest.raises(ValueError, match="current CUDA device"):
        B.it_residual_norm(d, torch.ones(2, 8), torch.ones(2, 8))
    with pytest.raises(ValueError, match="expected"):
        B.it_residual_norm(d, torch.ones(2, 8, dtype=torch.bfloat16), torch.ones(2, 8))
    r = B.RouteDesc(n_experts=4, top_k=2, logit_dtype=torch.float32)
    with pytest.raises(ValueError, match="current CUDA device"):
        B.it_route(r, torch.ones(2, 4), torch.zeros(2, 2, dtype=torch.int32), torch.ones(2, 2))
    with pytest.raises(KeyError):
        B.RouteDesc(n_experts=4, top_k=2, logit_dtype=torch.float32, score="tanh")
    with pytest.raises(ValueError, match="current CUDA device"):
        B.ExpertsDesc(n_experts=2, top_k=1, in_dim=8, out_dim=8, feat_dtype=torch.float32, W1=torch.ones(2, 8, 8))


@pytest.mark.parametrize("kw", [dict(in_dim=256, hidden_dim=1024, out_dim=256, top_k=1), dict(in_dim=64, hidden_dim=0, out_dim=4096, top_k=1, W2=None), dict(in_dim=64, hidden_dim=4096, out_dim=8),
                                dict(in_dim=768, hidden_dim=1024, out_dim=768, gated=1, top_k=4), dict(feat_dtype=0, in_dtype=0, in_dim=8, hidden_dim=2048, out_dim=8, top_k=1),
                                dict(feat_dtype=0, in_dtype=0, in_dim=1024, hidden_dim=1024, out_dim=1024, top_k=3), dict(in_dtype=2, in_dim=512, hidden_dim=1024, out_dim=256, top_k=1),
                                dict(in_dim=65536, hidden_dim=65536, out_dim=8, top_k=2)], ids=str)
@pytest.mark.parametrize("n_experts", [1, 4, 300, 1025])
def test_scratch_for_many_vertices_serves_fewer(kw, n_experts):
    """A program sizes its workspace once, for the most vertices that it scores at a time."""
    d = B.it_experts_desc(**{**dict(n_experts=n_experts, top_k=2, in_dim=64, hidden_dim=128, out_dim=64, feat_dtype=1, in_dtype=1, act=1, gated=0, W1=6 * BIG, b1=None, W2=7 * BIG,
                                    b2=None, w1_scale=None), **kw})
    before, size = 0, C.c_size_t()
    for n in [*range(0, 520), 700, 1000, 6143, 6145, 16384, 16385, 50_000, 60_000, 100_000, 1_000_000]:
        assert B.lib().it_experts_workspace_bytes(C.byref(d), n, C.byref(size)) == 0
        assert size.value >= before, n
        before = size.value


class _OnDevice:
    """What the binding asks of a tensor, with its answers set by the test."""

    def __init__(self, shape, dtype, address, device=0):
        import torch
        self.shape, self.dtype, self.address, self.device, self.dense = torch.Size(shape), dtype, address, device, True

    def get_device(self):
        return self.device

    def is_contiguous(self):
        return self.dense

    def data_ptr(self):
        return self.address

    def numel(self):
        return self.shape.numel()


def _descriptions(monkeypatch):
    """Every description with every tensor it may hold, each tensor's attribute and field, and the call that takes them (nothing is launched: no rows)."""
    import torch
    monkeypatch.setattr(B, "_device", lambda: 0)
    monkeypatch.setattr(B, "_stream_on", lambda device, stream: None)
    monkeypatch.setattr(B, "_nbytes", lambda t: 1 << 20)
    f32, bf16, e4m3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
    new = lambda shape, dtype: _OnDevice(shape, dtype, new.at.__next__())   # noqa: E731
    new.at = iter(range(1 << 30, 1 << 40, 1 << 24))
    norm = B.NormDesc(dim=64, feat_dtype=bf16, weight=new((64,), f32))
    route = B.RouteDesc(n_experts=8, top_k=2, logit_dtype=f32, balance_bias=new((8,), f32))
    experts = B.ExpertsDesc(n_experts=4, top_k=2, in_dim=64, hidden_dim=32, out_dim=16, feat_dtype=bf16, W1=new((4, 64, 32), e4m3), b1=new((4, 32), f32), W2=new((4, 32, 16), bf16),
                            b2=new((4, 16), f32), w1_scale=new((4, 32), f32))
    calls = {}

    class Library:
        def __getattr__(self, name):
            return lambda ref, *args: calls.__setitem__("c", ref._obj) or 0
    monkeypatch.setattr(B, "lib", lambda: Library())
    i32 = torch.int32
    return calls, [(norm, ["weight"], lambda: B.it_residual_norm(norm, new((3, 64), bf16), new((3, 64), bf16))),
                   (route, ["balance_bias"], lambda: B.it_route(route, new((3, 8), f32), new((3, 2), i32), new((3, 2), f32))),
                   (experts, ["W1", "b1", "W2", "b2", "w1_scale"],
                    lambda: B.it_experts_forward(experts, new((3, 64), e4m3), new((3, 2), i32), new((3, 2), f32), new((3, 16), bf16), new((1 << 20,), torch.uint8), x_scale=new((3,), f32)))]


def test_descriptions_follow_their_tensors(monkeypatch):
    """A tensor whose storage was replaced after the description was made: the call takes the new address, not the one that was given back."""
    calls, every = _descriptions(monkeypatch)
    for d, fields, call in every:
        call()
        for f in fields:
            t = getattr(d, f)
            assert getattr(calls["c"], f) == t.address
            t.address += 1 << 50
            call()
            assert getattr(calls["c"], f) == t.address, f


def test_descriptions_refuse_what_their_tensors_became(monkeypatch):
    """Another layout, size or device than the description says: refused by the call, as it would be by a new description."""
    import torch
    calls, every = _descriptions(monkeypatch)
    for d, fields, call in every:
        for f in fields:
            t = getattr(d, f)
            for name, value in (("dense", False), ("shape", torch.Size((3,))), ("device", 1)):
                was = getattr(t, name)
                setattr(t, name, value)
                if name == "device":   # (a tensor's address is another there)
                    t.address += 1 << 51
                with pytest.raises(ValueError):
                    call()
                setattr(t, name, was)
                call()


def test_descriptions_refuse_another_current_device(monkeypatch):
    """Made on one device, called on another: its tensors are not there, wherever the call's own are."""
    calls, every = _descriptions(monkeypatch)
    monkeypatch.setattr(B, "_device", lambda: 1)
    there = _OnDevice.__init__
    monkeypatch.setattr(_OnDevice, "__init__", lambda self, shape, dtype, address: there(self, shape, dtype, address, 1))
    for d, fields, call in every:
        with pytest.raises(ValueError, match="current CUDA device"):
            call()
