"""Edges of the training operators' host side (CPU: nothing here is launched)."""
import os
import subprocess
import sys

import pytest
import torch

from paper_2401_13660_gb300 import mbscan as mb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 1 << 40   # an aligned, never-dereferenced stand-in for a device address


def _at(i):
    return FAKE + (i << 34)


@pytest.mark.parametrize("n, vocab, width", [(0, 256, 64), (10, 0, 64), (10, 256, 0), (0, 256, 0), (10, 0, 0), (0, 0, 0)])
def test_embed_backward_workspace_of_nothing(n, vocab, width):
    # in a process of its own: what divides by a size ends it
    code = f"from paper_2401_13660_gb300 import mbscan as mb; print(mb.mb_embed_backward_workspace_size({n}, {vocab}, {width}))"
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT)
    assert r.returncode == 0 and int(r.stdout) >= 256, (r.returncode, r.stderr)
    need, lib = int(r.stdout), mb.load_library()
    call = lambda wb: lib.mb_embed_backward(_at(0), 0, _at(1), 0, 1.0, 1, _at(2), n, vocab, width, _at(3), wb, None)
    assert call(need) == mb.MB_OK   # nothing to add, so nothing is launched


def _cpu_calls():
    t, u = torch.zeros, torch.uint8
    x, w, tok = t(1, 2, 8), t(8, 4), t(2, dtype=u)
    ws = t(1 << 16, dtype=u)
    return dict(
        conv1d=lambda **k: mb.mb_conv1d(x, w, t(1, 2, 8), **k),
        conv1d_backward=lambda **k: mb.mb_conv1d_backward(x, w, t(1, 2, 8), **k),
        conv1d_backward_ws=lambda **k: mb.mb_conv1d_backward(x, w, x, grads=dict(dx=t(1, 2, 8), dw=t(8, 4)), ws=ws, **k),
        embed=lambda **k: mb.mb_embed(tok, t(4, 8), t(2, 8), **k),
        embed_backward=lambda **k: mb.mb_embed_backward(tok, t(2, 8), t(4, 8), **k),
        embed_backward_ws=lambda **k: mb.mb_embed_backward(tok, t(2, 8), t(4, 8), ws=ws, **k),
        cross_entropy=lambda **k: mb.mb_cross_entropy(t(2, 4), tok, t(2), **k),
        grad_norm=lambda **k: mb.mb_grad_norm([t(3)], **k),
        grad_norm_list=lambda **k: mb.mb_grad_norm(mb.mb_tensor_list([t(3)]), t(1), ws=ws, **k),
        grad_norm_empty=lambda **k: mb.mb_grad_norm([], t(1), **k),
        grad_clip=lambda **k: mb.mb_grad_clip([t(3)], t(1), 0.5, **k),
        grad_clip_out=lambda **k: mb.mb_grad_clip(mb.mb_tensor_list([t(3)]), t(1), 0.5, out=mb.mb_tensor_list([t(3)]), **k),
        grad_clip_empty=lambda **k: mb.mb_grad_clip([], t(1), 0.5, **k),
        rmsnorm=lambda **k: mb.mb_rmsnorm(t(1, 8), t(8), t(1, 8), **k),
        conv1d_step=lambda **k: mb.mb_conv1d_step(t(1, 8), t(1, 3, 8), w, t(1, 8), **k),
        prefill=lambda **k: mb.mb_scan_prefill(x, x, t(1, 2, 16), t(1, 2, 16), t(8, 16), t(1, 2, 8), **k),
        check=lambda **k: mb.mb_check(ws, **k))


@pytest.mark.parametrize("name", _cpu_calls())
@pytest.mark.parametrize("stream", [None, 0])
def test_host_tensors_are_refused(name, stream):
    # they agree with each other in every way; no launch may see their addresses
    with pytest.raises(ValueError, match="expected a CUDA device"):
        _cpu_calls()[name](stream=stream)


def test_a_workspace_that_grows_keeps_its_status():
    from paper_2401_13660_gb300.trainer import Workspace
    ws = Workspace("cpu")
    first = ws.get(300)
    first[:] = torch.arange(300, dtype=torch.int32).to(torch.uint8)
    assert ws.get(256) is first
    grown = ws.get(5000)
    assert grown is ws.buffer and grown.numel() >= 5000 and torch.equal(grown[:256], first[:256])


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("stand-in addresses: only where nothing can be launched")
    return mb.load_library()


def _lst(*entries):
    return (mb.mb_tensor * len(entries))(*(mb.mb_tensor(*e, 0) for e in entries))


def test_clipping_refuses_tensors_over_each_other(lib):
    F, B = mb.MB_F32, mb.MB_BF16
    run, bad = (mb.MB_OK, mb.MB_ERR_CUDA), mb.MB_ERR_INVALID_ARG

    def clip(entries, out=None):
        return lib.mb_grad_clip(_lst(*entries), None if out is None else _lst(*out), len(entries), _at(9), 1.0, None)
    two = [(_at(0), 10, F), (_at(1), 20, B)]
    away = [(_at(2), 10, F), (_at(3), 20, F)]
    assert clip(two) in run and clip(two, away) in run and clip(two, two) in run
    assert clip(two, [(_at(0), 10, F), (_at(3), 20, B)]) in run          # one in place, one not
    assert clip(two, [(_at(0) + 40, 10, F), (_at(1) + 40, 20, B)]) in run   # right behind the list
    assert clip(two, [away[0], (away[0][0] + 40, 20, F)]) in run            # right behind each other
    assert clip([(_at(0), 10, F), (_at(0), 10, F)], away[:1] + [(_at(3), 10, F)]) in run   # read twice, written apart
    assert clip([(None, 0, F), (_at(0), 0, F), *two], [(None, 0, F), (_at(0), 0, F), *two]) in run
    assert clip(two, [(_at(2), 10, F), (_at(0), 20, B)]) == bad             # over the list's other tensor
    assert clip(two, [(_at(1), 10, F), (_at(3), 20, F)]) == bad
    assert clip(two, [(_at(1) + 38, 10, F), (_at(3), 20, F)]) == bad        # its last element
    assert clip(two, [(_at(1), 10, F), (_at(0), 20, B)]) == bad             # changed about
    assert clip(two, [(_at(2), 10, F), (_at(2) + 36, 20, F)]) == bad        # over each other
    assert clip(two, [(_at(2), 10, F), (_at(2), 20, F)]) == bad
    assert clip([(_at(0), 10, F), (_at(0), 10, F)]) == bad                  # scaled twice, by two CTAs at once
    assert clip([(_at(0), 10, F), (_at(0) + 36, 10, F)]) == bad
    assert clip([(_at(0), 10, F), (_at(0) + 36, 10, F)], [(_at(0), 10, F), (_at(2), 10, F)]) == bad


@pytest.mark.parametrize("n", [3, 100, 101, 2500])
def test_clipping_finds_one_overlap_in_a_long_list(lib, n):
    # tensors of 16 elements, 64 bytes, packed; the outputs in another order
    ins = [(_at(0) + 64 * i, 16, mb.MB_F32) for i in range(n)]
    out = [(_at(1) + 64 * (i * 7919 % n), 16, mb.MB_F32) for i in range(n)]
    assert len({o[0] for o in out}) == n
    call = lambda o: lib.mb_grad_clip(_lst(*ins), None if o is None else _lst(*o), n, _at(9), 1.0, None)
    assert call(out) in (mb.MB_OK, mb.MB_ERR_CUDA) and call(None) in (mb.MB_OK, mb.MB_ERR_CUDA)
    for at, to in ((0, out[n - 1][0]), (n // 2, out[0][0] + 60), (n - 1, ins[0][0]), (1, ins[n - 1][0] + 4)):
        wrong = list(out)
        wrong[at] = (to, 16, mb.MB_F32)
        assert call(wrong) == mb.MB_ERR_INVALID_ARG


def test_clipping_accepts_outputs_between_the_list(lib):
    # gradients and their copies allocated in turn, one buffer per type, and both with the types mixed
    F, B, n = mb.MB_F32, mb.MB_BF16, 300
    call = lambda i, o: lib.mb_grad_clip(_lst(*i), _lst(*o), n, _at(9), 1.0, None)
    turn = [[(_at(0) + 128 * k + 64 * side, 16, F) for k in range(n)] for side in (0, 1)]
    types = [F if k % 3 else B for k in range(n)]
    flat = [(_at(1 if t == F else 2) + 64 * k, 16, t) for k, t in enumerate(types)]
    ins = [(_at(0) + 64 * k, 16, t) for k, t in enumerate(types)]
    for i, o in ((turn[0], turn[1]), (turn[1], turn[0][::-1]), (ins, flat), (flat, flat), (flat, ins), (ins[::-1], flat[::-1])):
        assert call(i, o) in (mb.MB_OK, mb.MB_ERR_CUDA)
        for at in (0, 7, n - 1):
            wrong = list(o)
            wrong[at] = (o[(at + 5) % n][0], 16, o[at][2])
            assert call(i, wrong) == mb.MB_ERR_INVALID_ARG
            wrong[at] = (i[(at + 5) % n][0] + 4, 12, o[at][2])
            assert call([(*x[:1], 12, x[2]) if k == at else x for k, x in enumerate(i)], wrong) == mb.MB_ERR_INVALID_ARG


def test_the_status_of_no_workspace():
    assert mb.mb_check(None, stream=0) == (mb.MB_ERR_INVALID_ARG, -1)
