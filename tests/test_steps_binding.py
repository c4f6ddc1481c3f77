"""CPU checks of what the binding of the rotary and norm calls takes for rows: a tensor whose rows are
one row of memory repeated is not dense."""
import pytest
import torch

from paper_2606_01774_gb300 import build, flare


@pytest.fixture(scope="module", autouse=True)
def here(request):
    """The library, which sees no rows and launches nothing; tensors count as on its device."""
    build.build()
    patch = pytest.MonkeyPatch()
    patch.setattr(flare, "_device", lambda: -1)
    yield
    patch.undo()


F32 = flare.FLARE_DT_F32
T, W, HEADS, D = 6, 64, 2, 64


def rows(*shape):
    return torch.zeros(shape)


def repeated(*shape):
    """As many rows, all of them the same memory."""
    return torch.zeros(shape[1:]).expand(shape)


def norm(**change):
    a = dict(x=rows(T, W), gate=rows(T, W), residual=rows(T, W), y=rows(T, W), h=rows(T, W))
    a.update(change)
    return flare.flare_block_norm(flare.block_norm_desc(0, W, F32), a["x"], a["gate"],
                                  a["residual"], None, None, a["y"], a["h"], stream=0)


def norm_bwd(**change):
    a = {k: rows(T, W) for k in "x gate residual dy dh dx dgate dresidual".split()}
    a.update(change)
    return flare.flare_block_norm_bwd(
        flare.block_norm_desc(0, W, F32), a["x"], a["gate"], a["residual"], None, None, a["dy"],
        a["dh"], a["dx"], a["dgate"], a["dresidual"], None, None, None, 0, stream=0)


TABLE, WORDS = torch.zeros(D // 2, dtype=torch.int64), torch.zeros(4, dtype=torch.int32)


def heads():
    return {k: rows(T, HEADS, D) for k in "q k v q_out k_out".split()}


def rotary(**change):
    a = heads()
    a.update(change)
    return flare.flare_rotary(flare.rotary_desc(0, 1, 0, HEADS, HEADS, D, D, F32), a["q"], a["k"],
                              TABLE, None, None, None, None, None, a["q_out"], a["k_out"], WORDS,
                              stream=0)


def append(**change):
    a = heads()
    a.update(change)
    pools = [rows(1, HEADS, 16, D) for _ in range(2)]
    return flare.flare_rotary_append_kv(
        flare.rotary_desc(0, 1, 0, HEADS, HEADS, D, D, F32, page_size=16, num_pages=1,
                          max_pages_per_req=1), a["q"], a["k"], a["v"], TABLE, None, WORDS, None,
        None, WORDS, a["q_out"], a["k_out"], *pools, WORDS, stream=0)


CALLS = [(norm, (T, W), "x gate residual y h"),
         (norm_bwd, (T, W), "x gate residual dy dh dx dgate dresidual"),
         (rotary, (T, HEADS, D), "q k q_out k_out"),
         (append, (T, HEADS, D), "q k v q_out k_out")]


@pytest.mark.parametrize("call,shape,name", [(c, s, n) for c, s, names in CALLS
                                             for n in names.split()])
def test_repeated_rows_are_refused(call, shape, name):
    assert call() == flare.FLARE_OK
    with pytest.raises(ValueError):
        call(**{name: repeated(*shape)})
    # one row is dense, however it is told
    assert call(**{name: repeated(1, *shape[1:])}) == flare.FLARE_OK


@pytest.mark.parametrize("call", [rotary, append])
def test_repeated_rows_and_heads_are_refused(call):
    same = rows(D).expand(T, HEADS, D)
    for name in "q k".split():
        with pytest.raises(ValueError):
            call(**{name: same})
        with pytest.raises(ValueError):  # the heads alone
            call(**{name: rows(T, 1, D).expand(T, HEADS, D)})
        part = repeated(T, HEADS, D)
        with pytest.raises(ValueError):  # in place
            call(**{name: part, name + "_out": part})
        with pytest.raises(ValueError):  # some of the leading dimensions
            call(**{name: rows(1, 3, HEADS, D).expand(2, 3, HEADS, D)})
