"""The policy update's binding and sizes without a GPU: what the host refuses before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2605_10875_amd import build, sol, synth


class _Calls:
    """The library with the entry points that would launch replaced: they note their arguments."""

    def __init__(self):
        self.seen = []
        real = sol.lib()
        for n in ("sol_policy_workspace_bytes", "sol_grad_clip_workspace_bytes"):
            setattr(self, n, getattr(real, n))
        for n in ("sol_policy_loss", "sol_grad_clip", "sol_adamw_step"):
            setattr(self, n, lambda *a, n=n: self.seen.append((n, a)) or 0)


@pytest.fixture
def ctx(monkeypatch):
    empty, zeros = torch.empty, torch.zeros
    monkeypatch.setattr(sol.torch.cuda, "current_device", lambda: -1)              # (what get_device() says of a host tensor)
    for name, fn in (("empty", empty), ("zeros", zeros)):
        monkeypatch.setattr(sol.torch, name, lambda *a, device=None, fn=fn, **k: fn(*a, **k))
    monkeypatch.setattr(sol, "_stream", lambda s: None)
    c = object.__new__(sol.Sol)
    c.cfg, c.handle, c.L = sol.make_cfg(synth.TINY, sol.F32, 16), C.c_void_p(), _Calls()
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


def test_row_steps():
    t = torch.zeros(2, 3, 4, 8)
    assert sol._row_step(t, "t") == 8
    assert sol._row_step(t[..., :5], "t") == 8                                     # padded rows
    assert sol._row_step(t[:, :, :, ::8], "t") == 8                                # one element per row
    assert sol._row_step(t[:1, :1, ::2, :5], "t") == 16                            # every second row
    assert sol._row_step(t[:1, :, :1, :5], "t") == 32
    assert sol._row_step(t[:1, :1, :1, :5], "t") == 5                              # one row
    assert sol._row_step(t[:0], "t") == 8
    for bad in (t.transpose(2, 3), t[..., ::2], t[:, ::2], t[:, :, :3], t.expand(2, 3, 4, 8)[:, :, :1].expand(2, 3, 4, 8)):
        with pytest.raises(ValueError):
            sol._row_step(bad, "t")


def test_policy_loss_hands_over_what_it_is_given(ctx):
    x, ids = _args()
    out = ctx.policy_loss(x, ids, clip=(0.1, 0.3), kl_coef=0.5, ref_logp=torch.zeros(2, 3, 4), mean="schedules")
    (name, a), = ctx.L.seen
    assert name == "sol_policy_loss" and a[1:5] == (x.data_ptr(), sol.F32, 5, ids.data_ptr()) and a[5:7] == (None, None) and a[7] is not None
    cfg = a[11]._obj
    assert (cfg.clip_low, cfg.clip_high, cfg.kl_coef, cfg.mean) == (0.1, 0.3, 0.5, 1) and a[12:16] == (2, 3, 4, 5)
    assert a[16:19] == (out["loss"].data_ptr(), out["stats"].data_ptr(), out["logp"].data_ptr()) and a[19] == out["grad"].data_ptr()
    assert out["logp"].shape == (2, 3, 4) and out["grad"].shape == x.shape and a[22] >= sol.lib().sol_policy_workspace_bytes(2, 3, 4)
    assert a[21] >= out["logp"].data_ptr() + 4 * 24                                # the workspace lies behind the outputs
    wide = torch.zeros(2, 3, 4, 16)[..., :5]                                       # padded rows
    out = ctx.policy_loss(wide, ids)
    assert ctx.L.seen[-1][1][3] == 16 and ctx.L.seen[-1][1][20] == 5 and out["grad"].is_contiguous()
    assert ctx.policy_loss(wide, ids, want_grad=False)["grad"] is None and ctx.L.seen[-1][1][19] is None


@pytest.mark.parametrize("change", [dict(logits=torch.zeros(2, 3, 4, 5, dtype=torch.float16)), dict(logits=torch.zeros(3, 4, 5)), dict(action_ids=None),
                                    dict(action_ids=torch.zeros(2, 3, 4, dtype=torch.int64)), dict(action_ids=torch.zeros(2, 3, 5, dtype=torch.int32)),
                                    dict(adv=torch.zeros(2, 3, 4, dtype=torch.float64)), dict(adv=torch.zeros(2, 4, 3).transpose(1, 2)),
                                    dict(old_logp=torch.zeros(2, 3)), dict(ref_logits=torch.zeros(2, 3, 4, 6)), dict(ref_logits=torch.zeros(2, 3, 4, 5, dtype=torch.bfloat16)),
                                    dict(eff=torch.zeros(2, 3, dtype=torch.int32)), dict(grad_out=torch.zeros(2, 3, 5, 4).transpose(2, 3)), dict(mean="rows"),
                                    dict(logits=torch.zeros(2, 3, 4, 10)[..., ::2])])
def test_policy_loss_refuses(ctx, change):
    x, ids = _args()
    with pytest.raises(ValueError):
        ctx.policy_loss(**{"logits": x, "action_ids": ids, **change})
    assert not ctx.L.seen


def test_lists_are_refused_with_the_tensor_that_is_wrong(monkeypatch):
    monkeypatch.setattr(sol.torch.cuda, "current_device", lambda: 0)
    good = torch.zeros(4)
    for lists, word in ((([good],), r"g\[0\]: not on the current device"), (([3],), r"g\[0\]: a tensor"), (([torch.zeros(2).double()],), r"g\[0\]: float32 or bf"),
                        (([good, torch.zeros(3, device="meta")],), r"g\[0\]: not on the current")):
        with pytest.raises(ValueError, match=word):
            sol._tensor_lists(lists, ("g",), (3,), 0)
    with pytest.raises(ValueError, match="same length"):
        sol._tensor_lists(([], [good]), ("a", "b"), (3, 3), 0)
    words, n = sol._tensor_lists(([], None, []), ("a", "b", "c"), (1, 1, 1), 2)
    assert n == 0 and len(words) == 0


def test_the_lists_are_compiled_with_the_library(tmp_path, monkeypatch):
    monkeypatch.setattr(build, "LISTS_LIB", str(tmp_path / "lists.so"))
    assert build.build_lists() == str(tmp_path / "lists.so") and (tmp_path / "lists.so").exists()
    before = (tmp_path / "lists.so").stat().st_mtime_ns
    build.build_lists(force=False)
    assert (tmp_path / "lists.so").stat().st_mtime_ns == before
