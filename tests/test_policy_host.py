"""The policy update's binding and sizes without a GPU: what the host refuses before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2605_10875_amd import build, sol, synth


LOSS = C.CFUNCTYPE(C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64,
                   C.c_void_p, C.POINTER(sol.PolicyCfg), C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                   C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p)
FIELDS = [f for f, _ in sol.PolicyCfg._fields_]


@pytest.fixture
def ctx(monkeypatch):
    """A binding whose entry point for the loss notes its arguments; host tensors stand for those of the device."""
    monkeypatch.setattr(sol.torch.cuda, "current_device", lambda: -1)              # (what get_device() says of a host tensor)
    monkeypatch.setattr(sol, "_stream", lambda s: C.c_void_p(0))
    c = object.__new__(sol.Sol)
    c.cfg, c.handle, c.L, c.seen = sol.make_cfg(synth.TINY, sol.F32, 16), C.c_void_p(), sol.lib(), []
    c.note = LOSS(lambda *a: c.seen.append(a[:11] + ({f: getattr(a[11].contents, f) for f in FIELDS},) + a[12:]) or 0)
    c._policy = (sol._native().policy_loss, sol._address(c.note), sol._address(c.L.sol_policy_workspace_bytes))
    return c


def _args(B=2, G=3, T=4, A=5, dtype=torch.float32):
    return torch.zeros(B, G, T, A, dtype=dtype), torch.zeros(B, G, T, dtype=torch.int32)


def test_null_context_and_sizes():
    L = sol.lib()
    assert L.sol_policy_loss(*[None, None, 0, 1] + [None] * 5 + [1, None, None, 1, 1, 1, 1] + [None] * 4 + [1, None, 0, None]) == sol.ERR_INVALID_ARG
    assert L.sol_grad_clip(None, None, 0, 1.0, 0.0, 1, None, None, None, 0, None) == sol.ERR_INVALID_ARG
    assert L.sol_adamw_step(None, None, 0, None, None, None, None, None) == sol.ERR_INVALID_ARG
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (-1, 1, 1)):
        assert L.sol_policy_workspace_bytes(*bad) == 0
    assert 0 < L.sol_policy_workspace_bytes(1, 1, 1) < L.sol_policy_workspace_bytes(1000, 1, 1)
    assert L.sol_grad_clip_workspace_bytes(-1) == 0
    assert 0 < L.sol_grad_clip_workspace_bytes(0) <= L.sol_grad_clip_workspace_bytes(240) < L.sol_grad_clip_workspace_bytes(2400)


def test_row_steps(ctx):
    t = torch.zeros(2, 3, 4, 8)

    def step(v):
        ctx.policy_loss(v, torch.zeros(v.shape[:3], dtype=torch.int32))
        return ctx.seen[-1][3]

    assert step(t) == 8
    assert step(t[..., :5]) == 8                                                   # padded rows
    assert step(t[:, :, :, ::8]) == 8                                              # one element per row
    assert step(t[:1, :1, ::2, :5]) == 16                                          # every second row
    assert step(t[:1, :, :1, :5]) == 32
    assert step(t[:1, :1, :1, :5]) == 5                                            # one row
    n = len(ctx.seen)
    for bad in (t.transpose(2, 3), t[..., ::2], t[:, ::2], t[:, :, :3], t[:, :, :1].expand(2, 3, 4, 8), t[:, :, :, :1].expand(2, 3, 4, 8)):
        with pytest.raises(ValueError):
            step(bad)
    assert len(ctx.seen) == n


def test_policy_loss_hands_over_what_it_is_given(ctx):
    x, ids = _args()
    out = ctx.policy_loss(x, ids, clip=(0.1, 0.3), kl_coef=0.5, ref_logp=torch.zeros(2, 3, 4), mean="schedules", temperature=1.3)
    a, = ctx.seen
    assert a[1:5] == (x.data_ptr(), sol.F32, 5, ids.data_ptr()) and a[5:7] == (None, None) and a[7] is not None and a[8:11] == (None, 0, None)
    assert a[11] == dict(clip_low=0.1, clip_high=0.3, kl_coef=0.5, entropy_coef=0.0, temperature=1.3, scale=1.0, mean=1) and a[12:16] == (2, 3, 4, 5)
    assert a[16:19] == (out["loss"].data_ptr(), out["stats"].data_ptr(), out["logp"].data_ptr()) and a[19] == out["grad"].data_ptr()
    assert out["loss"].shape == (1,) and out["stats"].shape == (4,) and out["logp"].shape == (2, 3, 4) and out["grad"].shape == x.shape
    assert a[22] == sol.lib().sol_policy_workspace_bytes(2, 3, 4) and a[21] == out["logp"].data_ptr() + 4 * 24
    room = out["loss"].untyped_storage()
    assert a[21] + a[22] <= room.data_ptr() + room.nbytes()                        # the workspace lies behind the outputs
    wide = torch.zeros(2, 3, 4, 16, dtype=torch.bfloat16)[..., :5]                 # padded rows
    out = ctx.policy_loss(wide, ids, ref_logits=wide.clone(), kl_coef=0.1)
    assert ctx.seen[-1][2:4] == (sol.BF16, 16) and ctx.seen[-1][9] == 5 and ctx.seen[-1][20] == 5 and out["grad"].is_contiguous()
    out = ctx.policy_loss(wide, ids, grad_out=wide)
    assert out["grad"] is wide and ctx.seen[-1][19:21] == (wide.data_ptr(), 16)
    assert ctx.policy_loss(wide, ids, want_grad=False)["grad"] is None and ctx.seen[-1][19] is None
    leaf = x.clone().requires_grad_(True)
    out = ctx.policy_loss(leaf, ids)
    assert not any(v.requires_grad for v in out.values())
    empty = ctx.policy_loss(x[:, :0], ids[:, :0])
    assert float(empty["loss"]) == 0.0 and empty["logp"].shape == (2, 0, 4) and empty["grad"].shape == (2, 0, 4, 5)


def test_a_status_of_the_loss_becomes_an_error(ctx):
    refuse = LOSS(lambda *a: sol.ERR_UNSUPPORTED)
    ctx._policy = ctx._policy[:1] + (sol._address(refuse),) + ctx._policy[2:]
    with pytest.raises(sol.SolError) as e:
        ctx.policy_loss(*_args())
    assert e.value.code == sol.ERR_UNSUPPORTED


@pytest.mark.parametrize("change", [dict(logits=torch.zeros(2, 3, 4, 5, dtype=torch.float16)), dict(logits=torch.zeros(3, 4, 5)), dict(action_ids=None),
                                    dict(action_ids=torch.zeros(2, 3, 4, dtype=torch.int64)), dict(action_ids=torch.zeros(2, 3, 5, dtype=torch.int32)),
                                    dict(adv=torch.zeros(2, 3, 4, dtype=torch.float64)), dict(adv=torch.zeros(2, 4, 3).transpose(1, 2)),
                                    dict(old_logp=torch.zeros(2, 3)), dict(ref_logits=torch.zeros(2, 3, 4, 6)), dict(ref_logits=torch.zeros(2, 3, 4, 5, dtype=torch.bfloat16)),
                                    dict(eff=torch.zeros(2, 3, dtype=torch.int32)), dict(grad_out=torch.zeros(2, 3, 5, 4).transpose(2, 3)), dict(mean="rows"),
                                    dict(logits=torch.zeros(2, 3, 4, 10)[..., ::2]),
                                    dict(logits=[1.0]), dict(adv=3), dict(logits=torch.zeros(2, 3, 4, 5).to_sparse())])
def test_policy_loss_refuses(ctx, change):
    x, ids = _args()
    with pytest.raises(ValueError):
        ctx.policy_loss(**{"logits": x, "action_ids": ids, **change})
    assert not ctx.seen


def _lists(*lists, types=None, typed=0, device=-1):
    names = tuple("abcdefgh"[:len(lists)])
    return sol._native().tensor_lists(lists, names, types or (3,) * len(lists), typed, device)


def test_lists_of_tensors_become_records():
    a, b = [torch.zeros(4), torch.zeros(2, 3)], (torch.zeros(4, dtype=torch.bfloat16), torch.zeros(6))
    words = memoryview(_lists(a, None, b, typed=2)).cast("q").tolist()
    assert words == [a[0].data_ptr(), 0, b[0].data_ptr(), 4, 1, a[1].data_ptr(), 0, b[1].data_ptr(), 6, 0]
    assert _lists([], None, []) == b""


@pytest.mark.parametrize("lists,types,word", [
    (([torch.zeros(4), 3],), (3,), r"a\[1\]: a tensor is needed"), (([torch.zeros(2).double()],), (3,), r"a\[0\]: float32 or bfloat16"),
    (([torch.zeros(2)], [torch.zeros(2)]), (1, 2), r"b\[0\]: bfloat16"), (([torch.zeros(4, 2).t()],), (3,), r"a\[0\]: has to be contiguous"),
    (([torch.zeros(4)], [torch.zeros(5)]), (1, 1), r"b\[0\]: not as many"), (([torch.zeros(4)], []), (1, 1), "same length"),
    (([torch.zeros(4).to_sparse()],), (3,), r"a\[0\]: not on")])
def test_lists_are_refused_with_the_tensor_that_is_wrong(lists, types, word):
    with pytest.raises(ValueError, match=word):
        _lists(*lists, types=types)
    with pytest.raises(ValueError, match="not on the current device"):
        _lists([torch.zeros(4)], device=0)
    with pytest.raises(TypeError):
        _lists(5)


def test_the_binding_is_compiled_with_the_library(tmp_path, monkeypatch):
    monkeypatch.setattr(build, "TORCH_LIB", str(tmp_path / "part.so"))
    assert build.build_torch() == str(tmp_path / "part.so")
    before = (tmp_path / "part.so").stat().st_mtime_ns
    build.build_torch(force=False)
    assert (tmp_path / "part.so").stat().st_mtime_ns == before


@pytest.mark.parametrize("grads,word", [([3], r"grads\[0\]: a tensor"), ([torch.zeros(2), torch.zeros(2).double()], r"grads\[1\]: float32 or bfloat16"),
                                        ([torch.zeros(4, 2).t()], r"grads\[0\]: has to be contiguous"), ([torch.zeros(2).to_sparse()], r"grads\[0\]: not on the current"),
                                        ([None], r"grads\[0\]: a tensor"), ((torch.zeros(2, device="meta"),), r"grads\[0\]: not on the current")])
def test_grad_clip_refuses(ctx, monkeypatch, grads, word):
    ctx._clip = None
    if grads[0] is not None and getattr(grads[0], "is_meta", False):
        monkeypatch.setattr(sol.torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match=word):
        ctx.grad_clip(grads, 1.0)
    with pytest.raises(TypeError):
        ctx.grad_clip(5, 1.0)
    with pytest.raises(TypeError):
        ctx.grad_clip([], "1")
