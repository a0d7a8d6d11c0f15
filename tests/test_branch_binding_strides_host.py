"""Masks and probabilities whose rows overlap (one row expanded to all, windows of one buffer): the binding describes them as they
lie, and the library refuses them before any launch.  (Host tensors; the library is asked only about what it has to refuse.)"""
import pytest
import torch

import paper_2602_15922_amd as w
from paper_2602_15922_amd import binding
from test_branch_binding_host import ARGS, F, I, R, T, V, WORDS

STRIDE = {"mask": "mask_stride", "p": "p_stride", "q": "q_stride"}
CALL = {"mask": "tree", "p": "verify", "q": "verify"}
FUNCTION = {"tree": "wam_attn_tree", "verify": "wam_verify_tree"}


def described(monkeypatch, call, **args):
    """The descriptor that a call hands to the library."""
    class Caught(Exception):
        pass

    class Lib:
        def __getattr__(self, name):
            def catch(desc, *_):
                raise Caught(name, desc._obj)
            return catch

    with monkeypatch.context() as m:
        m.setattr(binding, "lib", lambda: Lib())
        m.setattr(binding, "_stream_on", lambda stream, dev: None)
        f, rest = ARGS[call]
        with pytest.raises(Caught) as e:
            f(**{**rest(), **args})
    name, desc = e.value.args
    assert name == FUNCTION[call]
    return desc


def rows(name, kind):
    """[T, n] rows of a buffer that holds fewer than T * n entries."""
    make, n = (I, WORDS) if name == "mask" else (F, V)
    if kind == "expanded":
        return make(1, n).expand(T, n)
    return make(T + n - 1).as_strided((T, n), (1, 1))  # each row one entry past the last


@pytest.mark.parametrize("name", list(STRIDE))
@pytest.mark.parametrize("kind", ["expanded", "overlapping"])
def test_rows_that_overlap_are_refused(monkeypatch, name, kind):
    t = rows(name, kind)
    desc = described(monkeypatch, CALL[name], **{name: t})
    assert getattr(desc, STRIDE[name]) == t.stride(0) < t.shape[1]
    monkeypatch.setattr(binding, "_stream_on", lambda stream, dev: None)
    f, args = ARGS[CALL[name]]
    with pytest.raises(w.WamError, match="stride"):
        f(**{**args(), name: t})


@pytest.mark.parametrize("name", list(STRIDE))
def test_rows_apart_and_single_rows(monkeypatch, name):
    make, n = (I, WORDS) if name == "mask" else (F, V)
    assert getattr(described(monkeypatch, CALL[name]), STRIDE[name]) == n
    assert getattr(described(monkeypatch, CALL[name], **{name: make(T, n + 5)[:, :n]}), STRIDE[name]) == n + 5
    # one row: its stride says nothing
    one = make(1, n).as_strided((1, n), (0, 1))
    if name == "mask":
        args = dict(q=torch.zeros(1, 4, 128, dtype=torch.bfloat16), o=torch.zeros(1, 4, 128, dtype=torch.bfloat16), mask=one)
    else:
        args = dict(p=F(1, V), q=F(1, V), tokens=I(1), parent=I(1), u=F(1), path=I(1)) | {name: one}
    desc = described(monkeypatch, CALL[name], **args)
    assert desc.T == 1 and desc.R == R and getattr(desc, STRIDE[name]) == n


def test_one_column(monkeypatch):
    """Rows of a single entry may lie at any distance from 1 on."""
    assert described(monkeypatch, "tree", mask=I(1, T).t()).mask_stride == 1
    assert described(monkeypatch, "tree", mask=I(T, 7)[:, :1]).mask_stride == 7
    assert described(monkeypatch, "tree", mask=I(T, 0)).mask_words == 0
    assert described(monkeypatch, "verify", p=F(T, 3)[:, :1], q=F(1, T).t()).p_stride == 3
