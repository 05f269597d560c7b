"""What linear attention and the norms refuse, checked before any device is touched (no GPU needed)."""
import pytest
import struct

import torch

from paper_2603_09221_b200 import block, lqr

P = 1 << 20                 # an address that is never read: every call here is refused or only sized
INVALID, UNSUPPORTED = -1, -4


def _decay(**kw):
    a = dict(batch=2, tokens=8, offsets=0, heads=4, groups=2, dk=16, dv=32, dtype=1, softplus=1, scale=0.25, reserved=0)
    for n, at, width in (("q", 1, 32), ("k", 2, 32), ("v", 3, 128), ("delta", 4, 4), ("y", 5, 128)):
        a.update({n: at * P, n + "b": 8 * width, n + "t": width})
    a.update(A=P, delta_bias=P, state=0, state_out=0)
    a.update(kw)
    return block._DECAY_ARGS.pack(*a.values())


def _decay_grads(**kw):
    a = {}
    for n, at, width in (("dy", 6, 128), ("dq", 7, 32), ("dk", 8, 32), ("dv", 9, 128), ("ddelta", 10, 4)):
        a.update({n: at * P, n + "b": 8 * width, n + "t": width})
    a.update(dstate_out=0, dA=P, ddelta_bias=P, dstate=0)
    a.update(kw)
    return block._DECAY_GRADS.pack(*a.values())


def _norm(**kw):
    a = dict(rows=64, d=48, groups=4, dtype=1, eps=1e-6, x=P, z=2 * P, residual=3 * P, h=4 * P, y=5 * P, ldx=48, ldz=48, ldr=48, ldh=48, ldy=48, w_post=P, scale=P, w_pre=P)
    a.update(kw)
    return block._NORM_ARGS.pack(*a.values())


def _norm_grads(**kw):
    a = dict(dy=6 * P, dh=7 * P, dx=8 * P, dz=9 * P, dresidual=10 * P, lddy=48, lddh=48, lddx=48, lddz=48, lddr=48, dw_post=P, dscale=P, dw_pre=P)
    a.update(kw)
    return block._NORM_GRADS.pack(*a.values())


def _status(f, *args):
    status = f(*args)
    return status, lqr.load_library().ttc_lqr_last_error().decode()


@pytest.mark.parametrize("kw, status", [
    (dict(batch=-1), INVALID), (dict(tokens=-1), INVALID), (dict(heads=0), INVALID), (dict(groups=0), INVALID), (dict(groups=3), INVALID), (dict(dk=0), INVALID),
    (dict(dv=0), INVALID), (dict(dk=129), UNSUPPORTED), (dict(dv=129), UNSUPPORTED), (dict(dtype=0), INVALID), (dict(dtype=5), INVALID), (dict(q=0), INVALID), (dict(k=0), INVALID),
    (dict(v=0), INVALID), (dict(y=0), INVALID), (dict(A=0), INVALID), (dict(A=P + 2), INVALID), (dict(q=P + 1), INVALID), (dict(delta=P + 1), INVALID), (dict(kt=-32), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(y=P), INVALID), (dict(y=4 * P + 2), INVALID), (dict(y=3 * P + 64), INVALID),
    (dict(state=P, state_out=P + 64), INVALID), (dict(offsets=P + 2), INVALID), (dict(tokens=1 << 31), UNSUPPORTED), (dict(batch=1 << 20, tokens=1 << 20), UNSUPPORTED),
    (dict(heads=1 << 17, groups=1), UNSUPPORTED)])
def test_attention(kw, status):
    lib = block._load()
    assert _status(lib.ttc_decay_attention, 0, _decay(**kw), None, 0, None)[0] == status


def test_attention_step_gradients_and_workspaces():
    lib = block._load()
    assert _status(lib.ttc_decay_attention_step, 0, _decay(), None)[0] == INVALID                 # no state
    assert _status(lib.ttc_decay_attention_step, 0, _decay(state_out=P, dk=200), None)[0] == UNSUPPORTED
    need = lib.ttc_decay_attention_grad_workspace(0, _decay(), _decay_grads())
    assert need > 0
    for kw in (dict(dy=0), dict(dq=P), dict(dq=8 * P), dict(dv=6 * P), dict(ddelta=4 * P), dict(dA=P + 2), dict(dstate=P, dstate_out=P), dict(dkt=-1)):
        assert _status(lib.ttc_decay_attention_grad_workspace, 0, _decay(), _decay_grads(**kw))[0] == INVALID, kw
    for kw in (dict(), dict(ddelta=0)):
        assert _status(lib.ttc_decay_attention_grad_workspace, 0, _decay(delta=0), _decay_grads(**kw))[0] == INVALID
    assert lib.ttc_decay_attention_grad_workspace(0, _decay(delta=0), _decay_grads(ddelta=0, ddelta_bias=0)) > 0
    assert _status(lib.ttc_decay_attention_grad, 0, _decay(), _decay_grads(), P, need - 1, None)[0] == INVALID
    assert _status(lib.ttc_decay_attention_grad, 0, _decay(), _decay_grads(), P + 8, need, None)[0] == INVALID
    long = _decay(batch=1, tokens=1 << 16, heads=1, groups=1, y=1 << 40)                                      # in pieces
    assert lib.ttc_decay_attention_workspace(0, long) > 0
    status, text = _status(lib.ttc_decay_attention, 0, long, None, 0, None)
    assert status == INVALID and "workspace" in text


@pytest.mark.parametrize("kw, status", [
    (dict(rows=-1), INVALID), (dict(d=0), INVALID), (dict(groups=5), INVALID), (dict(groups=0), INVALID), (dict(dtype=4), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(x=0), INVALID), (dict(x=P + 1), INVALID), (dict(ldx=47), INVALID), (dict(ldz=47), INVALID), (dict(h=0, y=0, w_pre=0), INVALID), (dict(y=0), INVALID), (dict(w_pre=0), INVALID),
    (dict(w_post=0), INVALID), (dict(w_post=P + 2), INVALID), (dict(scale=P + 1), INVALID), (dict(h=P + 16), INVALID), (dict(y=3 * P + 32), INVALID), (dict(y=4 * P), INVALID),
    (dict(d=16385, groups=1, **{k: 16385 for k in ("ldx", "ldz", "ldr", "ldh", "ldy")}), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED)])
def test_norms(kw, status):
    lib = block._load()
    assert _status(lib.ttc_block_norm, 0, _norm(**kw), None)[0] == status


def test_gradients_of_norms():
    lib = block._load()
    need = lib.ttc_block_norm_grad_workspace(0, _norm(), _norm_grads())
    assert need > 0
    for kw in (dict(dy=0), dict(dx=P), dict(dz=4 * P), dict(dresidual=6 * P), dict(dz=8 * P), dict(lddx=47), dict(dw_pre=P + 2), dict(dresidual=7 * P + 32)):
        assert _status(lib.ttc_block_norm_grad_workspace, 0, _norm(), _norm_grads(**kw))[0] == INVALID, kw
    assert lib.ttc_block_norm_grad_workspace(0, _norm(), _norm_grads(dresidual=7 * P)) == need     # over dh
    for a, g in ((_norm(h=0), _norm_grads()), (_norm(z=0), _norm_grads()), (_norm(scale=0), _norm_grads()), (_norm(w_pre=0), _norm_grads(dw_pre=0)),
                 (_norm(w_post=0, groups=1), _norm_grads())):
        assert _status(lib.ttc_block_norm_grad_workspace, 0, a, g)[0] == INVALID
    assert lib.ttc_block_norm_grad_workspace(0, _norm(), _norm_grads(dw_post=0, dscale=0, dw_pre=0)) == 0
    assert _status(lib.ttc_block_norm_grad, 0, _norm(), _norm_grads(), P, need - 1, None)[0] == INVALID


def test_python_says_what_is_wrong():
    z = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t)  # noqa: E731
    q, v, A, f = z(2, 8, 2, 16), z(2, 8, 4, 32), z(4, t=torch.float32), torch.float32
    for args, kw, error in (((q, q, v, A), {}, ValueError), ((q, q, z(2, 8, 4, 32, t=f), A), {}, TypeError), ((q, z(2, 8, 2, 8), v, A), {}, ValueError),
                            ((q, q, v, z(3, t=f)), {}, ValueError), ((q, q, v, A), dict(delta=z(2, 8, 3)), ValueError), ((q, q, v, A), dict(delta_bias=A), ValueError),
                            ((q[0], q, v, A), {}, ValueError), ((q, q, v.transpose(2, 3).contiguous().transpose(2, 3), A), {}, ValueError),
                            ((q, q, v, A), dict(state=z(2, 4, 16, 31, t=f)), ValueError), ((q, q, v[0], A), {}, ValueError),
                            ((q[0], q[0], v[0], A), dict(offsets=z(3, t=torch.int64)), ValueError), ((z(2, 8, 2, 16, t=torch.float16), q, v, A), {}, ValueError)):
        with pytest.raises(error):
            block.decay_attention(*args, **kw)
    with pytest.raises(ValueError):                                                               # (no CPU way)
        block.decay_attention_step(q[:, 0], q[:, 0], v[:, 0], A, z(2, 4, 16, 32, t=f))
    with pytest.raises(ValueError):
        block.decay_attention_grad(v, q, q, v, A)
    x, w = z(4, 16), z(16, t=f)
    for kw, error in ((dict(x=x, w_pre=w), ValueError), (dict(x=x.double(), w_pre=w), TypeError), (dict(x=x, w_pre=z(15, t=f)), ValueError), (dict(x=x, w_pre=w, residual=z(3, 16)), ValueError),
                      (dict(x=x, z=z(4, 16, t=f)), ValueError), (dict(x=x, w_post=w, y=x), ValueError), (dict(x=x, w_pre=z(16)), ValueError)):
        with pytest.raises(error):
            block.block_norm(**kw)
    with pytest.raises(ValueError):
        block.block_norm_grad(x, dy=x, w_pre=w)


@pytest.mark.parametrize("record", ["_DECAY_ARGS", "_DECAY_GRADS", "_NORM_ARGS", "_NORM_GRADS"])
def test_a_module_built_for_other_records_is_not_used(monkeypatch, record):
    lib = block._load()
    assert block._short_way(lib) is not block._LongWay
    monkeypatch.setattr(block, record, struct.Struct(getattr(block, record).format + "q"))
    with pytest.warns(UserWarning, match="records"):
        assert block._short_way(lib) is block._LongWay
