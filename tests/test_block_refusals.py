"""What the operators of include/ttc_block.h refuse, checked before any device is touched (no GPU needed)."""
import pytest
import torch

from paper_2603_09221_b200 import block, lqr

P = 1 << 20                 # an address that is never read: every call here is refused or only sized


def _conv(**kw):
    a = dict(batch=2, tokens=8, offsets=0, d=16, taps=4, act=2, dtype=1, x=P, xb=128, xt=16, y=2 * P, yb=128, yt=16, w=P, bias=P, state=0, state_out=0)
    a.update(kw)
    return block._CONV_ARGS.pack(*a.values())


def _scan(**kw):
    a = dict(batch=2, tokens=8, offsets=0, d=16, n=16, groups=1, dtype=1, softplus=1, reserved=0)
    for k in ("x", "delta"):
        a.update({k: P, k + "b": 128, k + "t": 16})
    for k in ("B", "C"):
        a.update({k: P, k + "b": 128, k + "t": 16})
    a.update(z=0, zb=0, zt=0, y=2 * P, yb=128, yt=16, A=P, D=0, delta_bias=0, state=0, state_out=0)
    a.update(kw)
    return block._SCAN_ARGS.pack(*a.values())


def _linear(**kw):
    a = dict(rows=64, k=32, m=48, dtype=1, out_dtype=1, act=0, reserved=0, x=P, w=P, bias=0, residual=0, y=2 * P, pre=0,
             ldx=32, ldw=32, ldr=48, ldy=48, ldp=48)
    a.update(kw)
    return block._LINEAR_ARGS.pack(*a.values())


def _status(f, *args):
    status = f(*args)
    return status, lqr.load_library().ttc_lqr_last_error().decode()


INVALID, UNSUPPORTED = -1, -4


@pytest.mark.parametrize("kw, status", [
    (dict(batch=-1), INVALID), (dict(tokens=-1), INVALID), (dict(d=0), INVALID), (dict(taps=1), UNSUPPORTED), (dict(taps=5), UNSUPPORTED),
    (dict(act=3), UNSUPPORTED), (dict(act=9), UNSUPPORTED), (dict(dtype=7), INVALID), (dict(x=0), INVALID), (dict(y=0), INVALID), (dict(w=0), INVALID),
    (dict(x=P + 1), INVALID), (dict(w=P + 2), INVALID), (dict(xt=-16), INVALID), (dict(y=P), INVALID), (dict(y=P + 8), INVALID),
    (dict(tokens=1 << 31), UNSUPPORTED), (dict(batch=1 << 20, tokens=1 << 20), UNSUPPORTED), (dict(offsets=P + 2), INVALID)])
def test_convolution(kw, status):
    lib = block._load()
    assert _status(lib.ttc_causal_conv, 0, _conv(**kw), None)[0] == status


def test_convolution_step_and_gradients():
    lib = block._load()
    assert _status(lib.ttc_causal_conv_step, 0, _conv(), None)[0] == INVALID                     # no window
    grads = lambda **kw: block._CONV_GRADS.pack(*{**dict(dy=3 * P, dyb=128, dyt=16, dx=4 * P, dxb=128, dxt=16, dstate_out=0, dw=P, dbias=P, dstate=0), **kw}.values())  # noqa: E731
    assert lib.ttc_causal_conv_grad_workspace(0, _conv(), grads()) > 0
    for kw in (dict(dy=0), dict(dx=3 * P), dict(dx=P), dict(dw=P + 1), dict(dstate=P, dstate_out=P)):
        assert _status(lib.ttc_causal_conv_grad_workspace, 0, _conv(), grads(**kw))[0] == INVALID, kw
    status, text = _status(lib.ttc_causal_conv_grad, 0, _conv(), grads(), None, 0, None)
    assert status == INVALID and "workspace" in text
    status, text = _status(lib.ttc_causal_conv_grad, 0, _conv(), grads(), P + 8, 1 << 30, None)
    assert status == INVALID and "256" in text


@pytest.mark.parametrize("kw, status", [
    (dict(n=0), INVALID), (dict(n=129), UNSUPPORTED), (dict(groups=3), INVALID), (dict(groups=0), INVALID), (dict(d=0), INVALID), (dict(batch=-2), INVALID),
    (dict(dtype=3), INVALID), (dict(x=0), INVALID), (dict(delta=0), INVALID), (dict(B=0), INVALID), (dict(C=0), INVALID), (dict(A=0), INVALID),
    (dict(D=P + 1), INVALID), (dict(y=0), INVALID), (dict(y=P), INVALID), (dict(tokens=1 << 31), UNSUPPORTED), (dict(d=1 << 20), UNSUPPORTED)])
def test_scan(kw, status):
    lib = block._load()
    assert _status(lib.ttc_selective_scan, 0, _scan(**kw), None, 0, None)[0] == status


def test_scan_step_and_gradients():
    lib = block._load()
    assert _status(lib.ttc_selective_scan_step, 0, _scan(), None)[0] == INVALID                  # no state

    def grads(**kw):
        a = dict(dy=3 * P, dyb=128, dyt=16)
        for i, k in enumerate(("dx", "ddelta", "dB", "dC")):
            a.update({k: (4 + i) * P, k + "b": 128, k + "t": 16})
        a.update(dz=0, dzb=0, dzt=0, dstate_out=0, dA=P, dD=P, ddelta_bias=P, dstate=0)
        a.update(kw)
        return block._SCAN_GRADS.pack(*a.values())

    need = lib.ttc_selective_scan_grad_workspace(0, _scan(), grads())
    assert need > 0
    for kw in (dict(dy=0), dict(dx=3 * P), dict(dB=P), dict(dz=9 * P, dzt=16), dict(dA=P + 2)):
        assert _status(lib.ttc_selective_scan_grad_workspace, 0, _scan(), grads(**kw))[0] == INVALID, kw
    assert _status(lib.ttc_selective_scan_grad, 0, _scan(), grads(), P, need - 1, None)[0] == INVALID


def test_scan_of_few_channels_needs_a_workspace():
    lib = block._load()
    long = _scan(batch=1, tokens=4096)
    assert lib.ttc_selective_scan_workspace(0, long) > 0
    status, text = _status(lib.ttc_selective_scan, 0, long, None, 0, None)
    assert status == INVALID and "workspace" in text


@pytest.mark.parametrize("kw, status", [
    (dict(rows=-1), INVALID), (dict(k=0), INVALID), (dict(m=0), INVALID), (dict(dtype=0), INVALID), (dict(out_dtype=2), INVALID), (dict(act=5), INVALID),
    (dict(act=-1), INVALID), (dict(x=0), INVALID), (dict(w=0), INVALID), (dict(y=0), INVALID), (dict(x=P + 1), INVALID), (dict(bias=P + 2), INVALID),
    (dict(ldx=31), INVALID), (dict(ldw=31), INVALID), (dict(ldy=47), INVALID), (dict(residual=P, ldr=47), INVALID), (dict(rows=1 << 32), UNSUPPORTED), (dict(y=P), INVALID),
    (dict(pre=P + 16), INVALID)])
def test_linear(kw, status):
    lib = block._load()
    assert _status(lib.ttc_linear, 0, _linear(**kw), None, 0, None)[0] == status


def test_linear_gradients():
    lib = block._load()
    grads = lambda **kw: block._LINEAR_GRADS.pack(*{**dict(dy=3 * P, dx=4 * P, dw=5 * P, dbias=P, lddy=48, lddx=32, lddw=32), **kw}.values())  # noqa: E731
    assert lib.ttc_linear_grad_workspace(0, _linear(), grads()) >= 0
    for kw in (dict(dy=0), dict(lddy=47), dict(lddx=31), dict(lddw=31), dict(dbias=P + 1), dict(dx=P)):
        assert _status(lib.ttc_linear_grad_workspace, 0, _linear(), grads(**kw))[0] == INVALID, kw
    assert _status(lib.ttc_linear_grad_workspace, 0, _linear(act=2), grads())[0] == INVALID       # no pre


def test_linear_gradients_of_no_rows():
    """Every output there, by its address, and no rows: sums over nothing, and no product to plan (in a process of its own: a
    signal ends the process)."""
    import subprocess
    import sys
    code = """
from paper_2603_09221_b200 import block
from tests.test_block_refusals import P, _linear
lib = block._load()
for act, pre in ((0, 0), (2, 7 * P)):
    for out in (dict(dx=4 * P), dict(dw=5 * P), dict(dbias=6 * P), dict(dx=4 * P, dw=5 * P, dbias=6 * P)):
        g = dict(dy=3 * P, dx=0, dw=0, dbias=0, lddy=48, lddx=32, lddw=32)
        need = lib.ttc_linear_grad_workspace(0, _linear(rows=0, act=act, pre=pre), block._LINEAR_GRADS.pack(*{**g, **out}.values()))
        assert need >= 0, (out, need)
"""
    subprocess.run([sys.executable, "-c", code], check=True)


def test_outputs_that_overlap():
    lib = block._load()
    status = lambda f, *args: _status(getattr(lib, f), 0, *args)[0]  # noqa: E731
    # windows and states: in place or apart, not in part (one sequence's window is 3 x 16 x 2 bytes, its state 16 x 16 x 4)
    for out, want in ((6 * P + 96, INVALID), (6 * P - 2, INVALID)):
        assert status("ttc_causal_conv", _conv(state=6 * P, state_out=out), None) == want
    for out, want in ((6 * P + 1024, INVALID), (6 * P - 4, INVALID)):
        assert status("ttc_selective_scan", _scan(state=6 * P, state_out=out), None, 0, None) == want
    conv = lambda **kw: block._CONV_GRADS.pack(*{**dict(dy=3 * P, dyb=128, dyt=16, dx=4 * P, dxb=128, dxt=16, dstate_out=0, dw=P, dbias=P, dstate=0), **kw}.values())  # noqa: E731
    for out, want in ((6 * P, INVALID), (6 * P + 96, INVALID), (7 * P + 2, INVALID), (8 * P, True)):
        got = status("ttc_causal_conv_grad_workspace", _conv(state=6 * P), conv(dstate=out, dstate_out=7 * P))
        assert got == want or (want is True and got >= 0)

    def scan(**kw):
        a = dict(dy=3 * P, dyb=128, dyt=16, dx=4 * P, dxb=128, dxt=16)
        for k in ("ddelta", "dB", "dC", "dz"):
            a.update({k: 0, k + "b": 0, k + "t": 0})
        a.update(dstate_out=0, dA=0, dD=0, ddelta_bias=0, dstate=0)
        a.update(kw)
        return block._SCAN_GRADS.pack(*a.values())

    for out, want in ((6 * P, INVALID), (6 * P + 1024, INVALID), (7 * P + 4, INVALID), (8 * P, True)):
        got = status("ttc_selective_scan_grad_workspace", _scan(state=6 * P), scan(dstate=out, dstate_out=7 * P))
        assert got == want or (want is True and got >= 0)
    # matrices: y and pre with x, W and one another, y with parts of r; columns of one wider matrix are apart
    for kw, want in ((dict(w=5 * P, y=5 * P + 64), INVALID), (dict(w=5 * P, pre=5 * P - 2), INVALID), (dict(pre=2 * P + 32), INVALID),
                     (dict(residual=2 * P + 32), INVALID), (dict(residual=2 * P, ldr=64), INVALID), (dict(residual=2 * P), 0), (dict(residual=2 * P + 96, ldr=96, ldy=96), 0),
                     (dict(out_dtype=0, y=P + 4000), INVALID), (dict(out_dtype=0, pre=P, x=5 * P, y=P + 8), INVALID)):
        assert status("ttc_linear_workspace", _linear(**{**dict(w=9 * P), **kw})) == want, kw
    grads = lambda **kw: block._LINEAR_GRADS.pack(*{**dict(dy=3 * P, dx=4 * P, dw=5 * P, dbias=P, lddy=48, lddx=32, lddw=32), **kw}.values())  # noqa: E731
    for kw, want in ((dict(dx=3 * P), INVALID), (dict(dx=3 * P + 96, lddx=96, lddy=96), True), (dict(dx=9 * P), INVALID), (dict(dw=9 * P + 64), INVALID), (dict(dw=3 * P), INVALID),
                     (dict(dw=P), INVALID), (dict(dx=5 * P + 2), INVALID), (dict(dx=7 * P + 2), INVALID), (dict(), True)):
        got = status("ttc_linear_grad_workspace", _linear(w=9 * P, pre=7 * P, act=2), grads(**kw))
        assert got == want or (want is True and got >= 0), kw


def test_null_records():
    lib = block._load()
    for name in ("ttc_causal_conv", "ttc_causal_conv_step", "ttc_selective_scan_step"):
        assert getattr(lib, name)(0, None, None) == INVALID
    for name in ("ttc_selective_scan", "ttc_linear"):
        assert getattr(lib, name)(0, None, None, 0, None) == INVALID
        assert getattr(lib, name + "_workspace")(0, None) == INVALID


def test_binding_refuses_what_does_not_fit():
    x, w, b = torch.zeros(2, 5, 8, dtype=torch.bfloat16), torch.zeros(8, 4), torch.zeros(8)
    for bad, error in ((dict(w=torch.zeros(7, 4)), ValueError), (dict(bias=torch.zeros(8, dtype=torch.bfloat16)), ValueError),
                       (dict(act="tanh"), ValueError), (dict(x=x[0]), ValueError), (dict(x=x.double()), TypeError),
                       (dict(x=x.transpose(1, 2)), ValueError), (dict(state=torch.zeros(2, 4, 8, dtype=torch.bfloat16)), ValueError),
                       (dict(offsets=torch.zeros(3, dtype=torch.int32)), ValueError)):
        args = {**dict(x=x, w=w, bias=b, y=torch.empty_like(bad.get("x", x))), **bad}
        with pytest.raises(error):
            block.causal_conv(**args)
    r = torch.zeros(2, 5, 8)
    s = dict(x=r, delta=r, A=torch.zeros(8, 4), B=torch.zeros(2, 5, 4), C=torch.zeros(2, 5, 4), y=torch.empty_like(r))
    for bad in (dict(A=torch.zeros(8, 5)), dict(C=torch.zeros(2, 5, 2, 4)), dict(delta=r.bfloat16()), dict(B=torch.zeros(2, 4, 4)),
                dict(state=torch.zeros(2, 8, 5)), dict(D=torch.zeros(9)), dict(z=r[..., :4])):
        with pytest.raises(ValueError):
            block.selective_scan(**{**s, **bad})
    with pytest.raises(ValueError):                                  # nothing runs on the CPU
        block.selective_scan(**s)
    with pytest.raises(ValueError):
        block.linear(torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(3, 8, dtype=torch.bfloat16))


def test_records_are_laid_out_as_the_header_says(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "sizes.c"
    src.write_text("""#include <stddef.h>
#include <stdio.h>
#include "ttc_block.h"
#define END(t, last) (offsetof(t, last) + sizeof(((t*)0)->last))
int main(void) { printf("%zu %zu %zu %zu %zu %zu", END(ttc_conv_args, state_out), END(ttc_conv_grads, dstate), END(ttc_scan_args, state_out),
    END(ttc_scan_grads, dstate), END(ttc_linear_args, ldp), END(ttc_linear_grads, lddw)); return 0; }
""")
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), "-o", str(tmp_path / "sizes"), str(src)], check=True)
    sizes = [int(v) for v in subprocess.run([str(tmp_path / "sizes")], check=True, capture_output=True, text=True).stdout.split()]
    assert sizes == [s.size for s in (block._CONV_ARGS, block._CONV_GRADS, block._SCAN_ARGS, block._SCAN_GRADS, block._LINEAR_ARGS, block._LINEAR_GRADS)]


def test_every_declared_operator_is_bound():
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "ttc_block.h")).read(), flags=re.S)
    assert set(block.EXPORTS) == set(re.findall(r"\b(ttc_\w+)\s*\(", text))


def test_accesses_ask_for_no_more_than_sixteen_bytes(tmp_path):
    """The host sides let kernels read several elements at once where rows lie on 16 bytes; no such access may assume more."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "alignment.cu"
    src.write_text("""#include "block_common.cuh"
using namespace ttc::blk;
template <typename T> constexpr bool fits() {
    return alignof(Vec<T, 1>) == sizeof(T) && alignof(Vec<T, 2>) == 2 * sizeof(T) && alignof(Vec<T, 4>) <= 16 && alignof(Vec<T, 8>) <= 16 && sizeof(Vec<T, 8>) == 8 * sizeof(T);
}
static_assert(fits<float>() && fits<bf16>() && fits<__half>(), "");
""")
    subprocess.run(["nvcc", "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", os.path.join(root, "paper_2603_09221_b200", "csrc"), "-c",
                    "-o", str(tmp_path / "alignment.o"), str(src)], check=True)


def test_pieces_that_no_32_bits_count_are_refused():
    lib = block._load()
    a = block._SCAN_ARGS.pack((1 << 31) - (1 << 16), (1 << 31) - (1 << 16), P, 1, 1, 1, 0, 0, 0, *(P, 1, 1) * 4, *(0, 0, 0) * 2, P, 0, 0, 0, 0)
    g = block._SCAN_GRADS.pack(2 * P, 1, 1, *(0, 0, 0) * 5, 0, 0, 0, 0, 0)
    assert lib.ttc_selective_scan_grad_workspace(0, a, g) == UNSUPPORTED


def test_which_rows_overlap():
    """Outputs may lie in the same storage as inputs, in other columns, tokens or sequences; what is refused is rows that share an
    element (or rows of other strides whose ranges meet).  Against a count of the elements."""
    import random
    lib = block._load()
    rng = random.Random(3)

    def elements(at, batch, tokens, bs, ts, d):
        return {at + b * bs + t * ts + c for b in range(batch) for t in range(tokens) for c in range(d)}

    def refused(batch, tokens, d, x, xb, xt, y, yb, yt):
        a = _conv(batch=batch, tokens=tokens, d=d, dtype=0, x=P + 4 * x, xb=xb, xt=xt)
        g = block._CONV_GRADS.pack(64 * P, xb, xt, P + 4 * y, yb, yt, 0, 0, 0, 0)
        need = lib.ttc_causal_conv_grad_workspace(0, a, g)
        assert need == INVALID or need >= 0
        return need == INVALID

    assert not refused(2, 64, 16, 0, 128 * 16, 16, 64 * 16, 128 * 16, 16)           # the first tokens and the last ones of a batch
    assert refused(2, 65, 16, 0, 128 * 16, 16, 64 * 16, 128 * 16, 16)
    assert refused(2, 64, 16, 0, 128 * 16, 16, 16, 128 * 16, 16)                    # one token on
    assert not refused(1, 8, 16, 0, 0, 32, 16, 0, 32)                               # beside one another
    assert refused(4, 3, 16, 0, 64, 16, 48, 64, 16)                                 # three tokens of four, and on from the fourth into the next
    assert not refused(3, 8, 16, 0, 16, 96, 48, 16, 96)                             # [tokens, batch, channels], batches beside one another
    for _ in range(4000):
        batch, tokens, d = rng.randint(1, 4), rng.randint(1, 6), rng.randint(1, 5)
        strides = [rng.choice((0, 1, 2, 3, 5, 7, 10, 30, 31)) + rng.choice((0, 0, d, d * tokens)) for _ in range(2)]
        x, y = rng.randint(0, 60), rng.randint(0, 60)
        same = bool(elements(x, batch, tokens, *strides, d) & elements(y, batch, tokens, *strides, d))
        assert refused(batch, tokens, d, x, *strides, y, *strides) == same, (batch, tokens, d, x, y, strides)
