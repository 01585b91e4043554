"""Outputs of the rotation, attention and the clipped gradient that lie over other matrices of the call are refused; in place and next to each other they are not.  No GPU needed: every call here is refused, the
good ones for a workspace of no bytes, which is looked at last."""
import ctypes as C
import random

import pytest

import paper_2604_24708_amd as H
from paper_2604_24708_amd import binding as B
from test_lm_ops_heads_refusals import attention, attention_grad, clip, rotary, rotary_grad, rows, tensor

BASE = 1 << 40
OVER = "lies over"


def why(name, a):
    with pytest.raises(H.HdetError) as e:
        B._check(getattr(H.load_library(), name)(C.byref(a), None))
    assert e.value.code == H.HDET_EINVAL and name in H.hdet_last_error()
    return H.hdet_last_error()


def numbered(kw):
    return "-".join(f"{k}+{v.dev - BASE}/{v.row_stride}/{v.replica_stride}" if isinstance(v, B.hdet_rows) else f"{k}={v}" for k, v in kw.items()) or "as they are"


def at(place, row=64, rep=192):
    return rows(row, rep, BASE + place)


# q, k, q_out and k_out of two replicas of three rows, bfloat16: q | k of 64 + 32 columns in one matrix, the outputs in another
def slices(**kw):
    m = dict(q=at(0, 96, 288), k=at(128, 96, 288), q_out=at(4096, 96, 288), k_out=at(4224, 96, 288))
    m.update(kw)
    return m


@pytest.mark.parametrize("bad", [
    dict(k_out=at(4096, 96, 288)), dict(k_out=at(4160, 96, 288)), dict(q_out=at(128, 96, 288)), dict(q_out=at(0, 64, 192)), dict(q_out=at(2, 96, 288)), dict(q_out=at(64, 96, 288)),
    dict(q_out=at(0, 96, 320)), dict(k_out=at(0, 96, 288)), dict(k_out=at(126, 96, 288)), dict(k_out=at(188, 96, 288)), dict(q_out=at(576, 96, 288)), dict(q_out=at(64 - 576, 96, 288)),
    dict(k_out=at(128, 32, 288)), dict(k_out=at(4096, 32, 96)), dict(k_out=at(4096 + 192, 96, 288), q_out=at(4096 + 128, 96, 288))], ids=numbered)
def test_rotation(bad):
    assert OVER in why("hdet_head_rotary", rotary(**slices(**bad)))


def gradients(**kw):
    m = dict(q=at(0, 96, 288), k=at(256, 96, 288), dq_out=at(4096, 96, 288), dk_out=at(4352, 96, 288), dq=at(8192, 96, 288), dk=at(8448, 96, 288), workspace_bytes=0)
    m.update(kw)
    return m


@pytest.mark.parametrize("bad", [
    dict(dk=at(8192, 96, 288)), dict(dq=at(256, 96, 288)), dict(dq=at(4352, 96, 288)), dict(dk=at(4096, 96, 288)), dict(dk=at(0, 96, 288)), dict(dq=at(4096, 64, 192)), dict(dq=at(0, 64, 192)),
    dict(dq=at(4, 96, 288)), dict(dq=at(4096 + 252, 96, 288)), dict(dk=at(4352 - 4, 96, 288)), dict(dk=at(256 + 124, 96, 288))], ids=numbered)
def test_rotation_backward(bad):
    assert OVER in why("hdet_head_rotary_backward", rotary_grad(**gradients(**bad)))


@pytest.mark.parametrize("good", [
    dict(), dict(dq=at(4096, 96, 288), dk=at(4352, 96, 288)), dict(dq=at(0, 96, 288), dk=at(256, 96, 288)), dict(dq=at(0, 96, 288), dk=at(4352, 96, 288)),
    dict(rows=1, dq=at(4096, 64, 288)), dict(n_replicas=1, dq=at(4096, 96, 5000)), dict(dq=at(0, 96, 288), q_gain_dev=None, dq_gain_dev=None),
    dict(dk=at(8192 + 256, 96, 288))], ids=numbered)
def test_rotation_backward_in_place(good):
    a = rotary_grad(**gradients(**good))
    assert "workspace" in why("hdet_head_rotary_backward", a)


def test_attention():
    bf16 = dict(q=at(0, 128, 768), k=at(128, 128, 768), v=at(192, 128, 768))      # q | k | v of 64 + 32 + 32 columns, six rows (of ten keys) a replica
    for out in [at(0, 128, 768), at(128, 128, 768), at(2, 128, 768), at(-126, 128, 768), at(254, 128, 768), at(768 * 2, 128, 768)]:
        assert OVER in why("hdet_attention", attention(out=out, **bf16))
    f32 = dict(q=at(0, 128, 1280), k=at(256, 128, 1280), v=at(384, 128, 1280), out=at(1 << 20, 64, 384), dout=at(2 << 20, 64, 384), workspace_bytes=0)
    good = dict(dq=at(4 << 20, 128, 1280), dk=at((4 << 20) + 256, 128, 1280), dv=at((4 << 20) + 384, 128, 1280))
    assert "workspace" in why("hdet_attention_backward", attention_grad(**f32, **good))
    for bad in [dict(dk=at((4 << 20) + 252, 128, 1280)), dict(dv=at((4 << 20) + 256, 128, 1280)), dict(dv=at((4 << 20) + 380, 128, 1280)), dict(dq=at(0, 128, 1280)), dict(dk=at(4, 128, 1280)),
                dict(dk=at(384, 128, 1280)), dict(dq=at(1 << 20, 128, 1280)), dict(dq=at(1 << 20, 64, 384)), dict(dq=at((2 << 20) + 64, 64, 384)), dict(dv=at(1280 * 4 + 256, 128, 1280))]:
        assert OVER in why("hdet_attention_backward", attention_grad(**f32, **{**good, **bad}))


def test_strides_of_one_matrix_against_every_element():
    """dq against dk of the rotation in random places of one matrix of rows, or with replicas between each other's rows: refused if and only if an element is in both."""
    rng = random.Random(5)
    count = [0, 0]
    for _ in range(3000):
        n, length = rng.choice([1, 2, 3]), rng.choice([1, 2, 5])
        heads, k_heads, d = rng.choice([1, 2]), rng.choice([1, 3]), rng.choice([1, 2, 5])
        wide, narrow = heads * d, k_heads * d
        pitch = max(wide, narrow) + rng.choice([0, 0, 1, 4, 9])
        between = rng.random() < 0.3
        row, rep = (n * pitch, pitch) if between else (pitch, length * pitch + rng.choice([0, 3]))
        shift = rng.randrange(-2 * n * length * pitch, 2 * n * length * pitch)
        one, other = ({(z * rep + i * row + c + s) for z in range(n) for i in range(length) for c in range(w)} for w, s in ((wide, 0), (narrow, shift)))
        far = 1 << 24
        a = rotary_grad(n_replicas=n, rows=length, head_dim=d, rotated=0, q_heads=heads, k_heads=k_heads, q=at(far, row, rep), k=at(2 * far, row, rep), dq_out=at(3 * far, row, rep),
                        dk_out=at(4 * far, row, rep), dq=at(8 * far, row, rep), dk=at(8 * far + 4 * shift, row, rep), workspace_bytes=0)
        meets = bool(one & other)
        assert (OVER if meets else "workspace") in why("hdet_head_rotary_backward", a), (n, length, wide, narrow, row, rep, shift)
        count[meets] += 1
    assert min(count) > 500


def places(grad, out, **kw):
    return tensor(grad=grad, out=out if out is not None else rows(0, 0, None), **kw)


HERE, THERE, FAR = at(0, 7, 21), at(4096, 7, 21), at(8192, 7, 21)
BF16 = dict(dtype=H.HDET_TYPE_BF16)


@pytest.mark.parametrize("bad", [
    # an output where another tensor's gradient starts, whichever comes first, and a gradient that is scaled in place and read by another tensor
    [places(HERE, THERE), places(FAR, HERE)], [places(FAR, HERE), places(HERE, THERE)], [places(HERE, None), places(HERE, THERE)], [places(HERE, THERE, **BF16), places(FAR, HERE)],
    [places(HERE, THERE), places(HERE, HERE)],
    # an output over its own gradient, of other types, strides or a part of it
    [places(HERE, HERE, **BF16)], [places(HERE, at(0, 8, 24))], [places(HERE, at(0, 7, 22))], [places(HERE, at(4, 7, 21))], [places(HERE, at(-4, 7, 21))], [places(HERE, at(4 * 41, 7, 21))]])
def test_clipped_gradients(bad):
    message = why("hdet_clip_gradients", clip(bad))
    assert OVER in message or "written where another" in message


@pytest.mark.parametrize("good", [
    [places(HERE, HERE)], [places(HERE, at(4 * 42, 7, 21))], [places(HERE, at(0, 9, 21), rows=1)], [places(HERE, None)], [places(HERE, None, **BF16)],
    [places(HERE, THERE), places(HERE, FAR)],                   # one gradient twice, read alone
    [places(at(0, 7, 42), at(4096, 7, 42)), places(at(84, 7, 42), at(4096 + 84, 7, 42))], [places(HERE, THERE), places(FAR, FAR), places(at(1 << 20, 7, 21), None)],
    [places(HERE, THERE), places(FAR, HERE, rows=0)]])
def test_clipped_gradients_in_place_and_apart(good):
    assert "workspace" in why("hdet_clip_gradients", clip(good, workspace_bytes=0))
