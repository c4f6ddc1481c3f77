"""CPU checks of the rotary, logits and norm calls' host side: every refusal happens before any
CUDA work.  The pointers are stand-ins on the right boundaries; no call gets past its checks,
except those on nothing, which launch nothing."""
import ctypes

import pytest
import torch

from paper_2606_01774_gb300 import build, flare

OK, BAD, NO = flare.FLARE_OK, flare.FLARE_ERR_INVALID_ARGUMENT, flare.FLARE_ERR_UNSUPPORTED
AT = 0x10000  # 256-byte aligned, never read


@pytest.fixture(scope="module")
def lib():
    build.build()
    return flare.load()


def changed(d, kw):
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def rotary(**kw):
    return changed(flare.rotary_desc(2, 4, 8, 16, 2, 256, 64, flare.FLARE_DT_BF16, page_size=64,
                                     num_pages=10, max_pages_per_req=5), kw)


def freq(**kw):
    return changed(flare.rotary_freq_desc(64, 1e4, flare.FLARE_ROTARY_BY_PARTS, 4.0, 4096.0), kw)


def logits(**kw):
    return changed(flare.tree_logits_desc(2, 4, 1000, flare.FLARE_DT_BF16, 16, 4), kw)


def norm(**kw):
    return changed(flare.block_norm_desc(8, 1024, flare.FLARE_DT_BF16, group=128), kw)


# every array far from every other
NAMES = {
    "flare_rotary": "q k table position prefix_len token_len parent token_start q_out k_out "
                    "dev_status",
    "flare_rotary_append_kv": "q k v table position prefix_len token_len token_start page_table "
                              "q_out k_out k_pool v_pool dev_status",
    "flare_tree_logits": "logits history history_len output_start token parent node_len repetition "
                         "presence frequency bias_token bias_value bias_len mask out dev_status",
    "flare_block_norm": "x gate residual post_weight pre_weight y h",
    "flare_block_norm_bwd": "x gate residual post_weight pre_weight dy dh dx dgate dresidual "
                            "dpost_weight dpre_weight workspace workspace_bytes",
}
DESC = {"flare_rotary": rotary, "flare_rotary_append_kv": rotary, "flare_tree_logits": logits,
        "flare_block_norm": norm, "flare_block_norm_bwd": norm}
# a call that all checks accept leaves these out, having the others
LEFT_OUT = {"flare_rotary": {"token_start"}, "flare_rotary_append_kv": {"token_start"}}


def run(lib, call, desc=None, **change):
    d = DESC[call]() if desc is None else desc
    names = NAMES[call].split()
    assert all(k in names for k in change)
    values = []
    for i, n in enumerate(names):
        v = None if n in LEFT_OUT.get(call, ()) else (1 << 30 if n == "workspace_bytes"
                                                      else AT + (i << 32))
        values.append(change.get(n, v))
    return getattr(lib, call)(ctypes.byref(d), *values, None)


NEEDED = {
    "flare_rotary": "table dev_status q_out k_out",
    "flare_rotary_append_kv": "k v table prefix_len page_table q_out k_pool v_pool dev_status",
    "flare_tree_logits": "logits history_len parent node_len bias_token bias_value bias_len out "
                         "dev_status",
    "flare_block_norm": "x h",
    "flare_block_norm_bwd": "x dh dx dgate workspace",
}


@pytest.mark.parametrize("call", sorted(NAMES))
def test_needed_pointers(lib, call):
    for name in NEEDED[call].split():
        assert run(lib, call, **{name: None}) == BAD, name
    assert getattr(lib, call)(None, *[AT] * len(NAMES[call].split()), None) == BAD


def test_pointers_that_go_together(lib):
    assert run(lib, "flare_rotary", q=None, k=None, q_out=None, k_out=None) == BAD
    assert run(lib, "flare_rotary", q=None) == BAD
    for extra in ("token_len", "parent"):
        other = "parent" if extra == "token_len" else "token_len"
        assert run(lib, "flare_rotary", token_start=AT, **{other: None}) == BAD
    assert run(lib, "flare_rotary_append_kv", token_start=AT) == BAD
    assert run(lib, "flare_block_norm", norm(pre_norm=0)) == BAD  # an h that is none
    assert run(lib, "flare_block_norm", norm(pre_norm=0), h=None, y=None) == BAD
    assert run(lib, "flare_block_norm_bwd", norm(pre_norm=0), dh=None) == BAD  # dpre_weight
    assert run(lib, "flare_block_norm_bwd", norm(post_norm=0)) == BAD
    assert run(lib, "flare_block_norm_bwd", gate=None) == BAD
    assert run(lib, "flare_block_norm_bwd", residual=None) == BAD
    assert run(lib, "flare_block_norm_bwd", norm(pre_norm=0), dh=None, dy=None,
               dpre_weight=None) == BAD


def test_alignment(lib):
    for call, names in (("flare_rotary", "q k q_out k_out"),
                        ("flare_rotary_append_kv", "q k v q_out k_out k_pool v_pool"),
                        ("flare_block_norm", "x gate residual post_weight pre_weight y h"),
                        ("flare_block_norm_bwd", "x gate residual post_weight pre_weight dy dh dx "
                                                 "dgate dresidual workspace")):
        for n in names.split():
            assert run(lib, call, **{n: AT + (50 << 32) + 8}) == BAD, (call, n)
    assert run(lib, "flare_rotary", table=AT + 4) == BAD
    assert run(lib, "flare_tree_logits", logits=AT + 1) == BAD
    assert run(lib, "flare_tree_logits", logits(logits_dtype=flare.FLARE_DT_F32), out=AT + 2) == BAD
    assert run(lib, "flare_block_norm_bwd", dpost_weight=AT + 2) == BAD


def test_overlaps(lib):
    # in place is fine on nothing; a shifted copy of the input's rows is not
    assert run(lib, "flare_rotary", rotary(num_requests=0), q=AT, q_out=AT) == OK
    assert run(lib, "flare_rotary", q=AT, q_out=AT + 512) == BAD
    assert run(lib, "flare_rotary", k=AT + 512, k_out=AT) == BAD
    assert run(lib, "flare_rotary_append_kv", k=AT + 512, k_out=AT) == BAD
    assert run(lib, "flare_tree_logits", logits=AT, out=AT + 16) == BAD
    assert run(lib, "flare_tree_logits", logits=AT + 2 * 2 * 4 * 1000 - 2, out=AT) == BAD
    assert run(lib, "flare_block_norm", y=AT, h=AT) == BAD
    assert run(lib, "flare_block_norm", norm(x_stride=2048), x=AT, y=AT) == BAD


def test_overlaps_of_rows(lib):
    """Every pair of an output and another array that share bytes but are not the same rows."""
    wide, rows = 1024 * 2, 8  # of norm()
    at = lambda call, n: AT + (NAMES[call].split().index(n) << 32)  # noqa: E731
    outs = {"flare_block_norm": ("y h", "x gate residual"),
            "flare_block_norm_bwd": ("dx dgate dresidual", "x gate residual dy dh")}
    for call, (outputs, inputs) in outs.items():
        for o in outputs.split():
            for i in inputs.split() + [n for n in outputs.split() if n != o]:
                for off in (16, -16, wide * (rows - 1)):
                    assert run(lib, call, **{o: at(call, i) + off}) == BAD, (call, o, i)
            for i in outputs.split():
                if i != o:
                    assert run(lib, call, **{o: at(call, i)}) == BAD, (call, o, i)
    # rows of one stride between each other: fine while none reaches into another's
    d = norm(x_stride=2048, gate_stride=2048)
    a = at("flare_block_norm_bwd", "dx")
    for off in (wide - 16, 16, 2 * wide - 16):
        assert run(lib, "flare_block_norm_bwd", d, dgate=a + off) == BAD
    assert run(lib, "flare_block_norm_bwd", norm(x_stride=2048, gate_stride=4096),
               dgate=a + wide) == BAD
    assert run(lib, "flare_block_norm_bwd", d, dgate=a + wide, workspace=None) == BAD
    for call in ("flare_rotary", "flare_rotary_append_kv"):
        assert run(lib, call, q_out=at(call, "k")) == BAD  # another input's place
        assert run(lib, call, k_out=at(call, "q")) == BAD
        assert run(lib, call, k_out=at(call, "q_out") + 16) == BAD
    call = "flare_rotary_append_kv"
    for i in "q k v q_out k_out v_pool".split():
        assert run(lib, call, k_pool=at(call, i)) == BAD, i
    assert run(lib, call, v_pool=at(call, "k_pool") + 1024) == BAD


def test_alignment_of_small_arrays(lib):
    for call, names in (("flare_rotary", "position prefix_len token_len parent dev_status"),
                        ("flare_rotary_append_kv", "position prefix_len page_table dev_status"),
                        ("flare_tree_logits", NAMES["flare_tree_logits"])):
        for n in names.split():
            if n not in ("logits", "out"):
                assert run(lib, call, **{n: AT + (50 << 32) + 2}) == BAD, (call, n)


@pytest.mark.parametrize("change,status", [
    (dict(num_requests=-1), BAD), (dict(block_len=0), BAD), (dict(num_q_heads=0), BAD),
    (dict(num_kv_heads=0), BAD), (dict(act_dtype=2), BAD), (dict(layout=2), BAD),
    (dict(inverse=2), BAD), (dict(amplitude=float("nan")), BAD),
    (dict(amplitude=float("inf")), BAD), (dict(head_dim=96), NO), (dict(rotary_dim=8), NO),
    (dict(rotary_dim=72), NO), (dict(rotary_dim=272), NO), (dict(q_stride=4095), BAD),
    (dict(q_stride=4100), BAD), (dict(k_stride=511), BAD), (dict(v_stride=516), BAD),
    (dict(k_stride=1 << 32), NO), (dict(num_requests=1 << 20, block_len=1 << 20), NO)])
def test_rotary_shapes(lib, change, status):
    for call in ("flare_rotary", "flare_rotary_append_kv"):
        assert run(lib, call, rotary(**change)) == status
    if "block_len" not in change:  # packed rows
        assert run(lib, "flare_rotary", rotary(**change), token_start=AT, token_len=None,
                   parent=None) == status


def test_rotary_more_shapes(lib):
    assert run(lib, "flare_rotary", rotary(block_len=65)) == NO  # a tree's nodes
    assert run(lib, "flare_rotary", rotary(num_tokens=-1), token_start=AT, token_len=None,
               parent=None) == BAD
    for change, status in ((dict(page_size=0), BAD), (dict(page_size=48), NO),
                           (dict(num_pages=-1), BAD), (dict(max_pages_per_req=-1), BAD),
                           (dict(max_pages_per_req=1 << 19), NO)):
        assert run(lib, "flare_rotary_append_kv", rotary(**change)) == status


@pytest.mark.parametrize("change,status", [
    (dict(rotary_dim=8), NO), (dict(rotary_dim=264), NO), (dict(rotary_dim=40), NO),
    (dict(scaling=4), BAD), (dict(base=0.5), BAD), (dict(base=float("nan")), BAD),
    (dict(factor=0.0), BAD), (dict(factor=float("inf")), BAD), (dict(original_len=0.0), BAD),
    (dict(low_turns=-1.0), BAD), (dict(low_turns=32.0), BAD), (dict(high_turns=float("inf")), BAD)])
def test_tables(lib, change, status):
    assert lib.flare_rotary_table(ctypes.byref(freq(**change)), AT, None) == status
    assert lib.flare_rotary_table(ctypes.byref(freq()), AT + 4, None) == BAD
    assert lib.flare_rotary_table(ctypes.byref(freq()), None, None) == BAD
    assert lib.flare_rotary_table(None, AT, None) == BAD


@pytest.mark.parametrize("change,status", [
    (dict(num_requests=-1), BAD), (dict(num_nodes=0), BAD), (dict(num_nodes=65), NO),
    (dict(vocab_size=0), BAD), (dict(vocab_size=(1 << 24) + 1), NO), (dict(logits_dtype=3), BAD),
    (dict(max_history=-1), BAD), (dict(max_history=(1 << 24) + 1), NO), (dict(max_bias=-1), BAD),
    (dict(max_bias=65537), NO), (dict(num_requests=1 << 30, vocab_size=1 << 24), NO)])
def test_logits_shapes(lib, change, status):
    # in place: the sizes of the last case would overlap anything
    assert run(lib, "flare_tree_logits", logits(**change), logits=AT, out=AT) == status


@pytest.mark.parametrize("change,status", [
    (dict(num_tokens=-1), BAD), (dict(width=0), BAD), (dict(width=1020), NO),
    (dict(width=16392), NO), (dict(group=-1), BAD), (dict(group=32), NO),
    (dict(group=256, width=1088), BAD), (dict(shared_weight=2), BAD), (dict(post_norm=2), BAD),
    (dict(pre_norm=-1), BAD), (dict(gate_act=3), BAD), (dict(act_dtype=7), BAD),
    (dict(eps=0.0), BAD), (dict(eps=float("nan")), BAD), (dict(residual_scale=float("inf")), BAD),
    (dict(x_stride=1016), BAD), (dict(gate_stride=1028), BAD), (dict(x_stride=1 << 40), NO)])
def test_norm_shapes(lib, change, status):
    n = ctypes.c_size_t(0)
    assert run(lib, "flare_block_norm", norm(**change)) == status
    assert run(lib, "flare_block_norm_bwd", norm(**change)) == status
    assert lib.flare_block_norm_bwd_workspace_size(ctypes.byref(norm(**change)),
                                                   ctypes.byref(n)) == status


def test_norm_workspace(lib):
    need = flare.flare_block_norm_bwd_workspace_size(norm())
    assert need > 0
    assert run(lib, "flare_block_norm_bwd", workspace_bytes=need - 1) == BAD
    assert lib.flare_block_norm_bwd_workspace_size(ctypes.byref(norm()), None) == BAD
    assert flare.flare_block_norm_bwd_workspace_size(norm(num_tokens=0)) == 0
    # without weight gradients none is needed, and nothing is launched on no rows
    assert run(lib, "flare_block_norm_bwd", norm(num_tokens=0), workspace=None, workspace_bytes=0,
               dpost_weight=None, dpre_weight=None) == OK


def test_calls_on_nothing_launch_nothing(lib):
    before = flare.flare_launch_count()
    assert run(lib, "flare_rotary", rotary(num_requests=0)) == OK
    assert run(lib, "flare_rotary_append_kv", rotary(num_requests=0)) == OK
    assert run(lib, "flare_rotary", rotary(num_tokens=0), token_start=AT, token_len=None,
               parent=None) == OK
    assert run(lib, "flare_tree_logits", logits(num_requests=0)) == OK
    assert run(lib, "flare_block_norm", norm(num_tokens=0)) == OK
    # an array of no rows may be a null pointer
    assert run(lib, "flare_rotary", rotary(num_requests=0), q=None, k=None, q_out=None) == OK
    assert run(lib, "flare_tree_logits", logits(num_requests=0), logits=None) == OK
    assert run(lib, "flare_block_norm", norm(num_tokens=0), x=None, y=None) == OK
    assert flare.flare_launch_count() == before


def test_short_conv_still_takes_its_own_activations(lib):
    d = flare.conv_desc(1, 4, 64, 4, 2, flare.FLARE_DT_BF16, flare.FLARE_ACT_SIGMOID)
    assert lib.flare_short_conv(ctypes.byref(d), *[AT] * 8, None) == BAD


def test_the_binding_refuses_other_strides_and_devices(monkeypatch):
    here = torch.zeros(4, 16, 256)
    status = torch.zeros(1, dtype=torch.int32)
    table = torch.zeros(32, dtype=torch.int64)
    d = rotary(num_requests=0, act_dtype=flare.FLARE_DT_F32, q_stride=0)

    def call(q=here, out=None, desc=d):
        return flare.flare_rotary(desc, q, None, table, None, None, None, None, None,
                                  torch.zeros(4, 16, 256) if out is None else out, None, status,
                                  stream=0)

    monkeypatch.setattr(flare, "_device", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        call()
    monkeypatch.setattr(flare, "_device", lambda: -1)  # where these tensors are
    assert call() == OK
    wide = torch.zeros(4, 20, 256)
    with pytest.raises(ValueError, match="strides"):
        call(wide[:, :16])
    with pytest.raises(ValueError, match="strides"):
        call(here.transpose(1, 2).contiguous().transpose(1, 2))
    with pytest.raises(ValueError):
        call(out=wide[:, :16])
    s = rotary(num_requests=0, act_dtype=flare.FLARE_DT_F32, q_stride=20 * 256)
    assert call(wide[:, :16], desc=s) == OK
    assert call(wide[:, :16], wide[:, :16], desc=s) == OK  # in place
    assert call(wide.view(2, 2, 20, 256)[:, :, :16], desc=s) == OK
    with pytest.raises(ValueError, match="strides"):
        call(here, desc=s)
    n = norm(num_tokens=0, act_dtype=flare.FLARE_DT_F32, x_stride=2048)
    x = torch.zeros(3, 2048)
    with pytest.raises(ValueError, match="strides"):
        flare.flare_block_norm(n, x[:, ::2], None, None, None, None, None, x, stream=0)
    assert flare.flare_block_norm(n, x[:, :1024], None, None, None, None, None, x.clone(),
                                  stream=0) == OK


def test_row_counts_up_to_the_last_int(lib):
    """The workspace of 2^31 - 1 rows is that of 2^30: the launch has as many CTAs as the SMs hold."""
    for width in (8, 64, 1024, 4096, 16384):
        for dtype in (flare.FLARE_DT_BF16, flare.FLARE_DT_F32):
            for pre in (0, 1):
                need = [flare.flare_block_norm_bwd_workspace_size(
                    flare.block_norm_desc(t, width, dtype, pre_norm=pre))
                    for t in (1 << 30, (1 << 31) - 8, (1 << 31) - 1)]
                assert need[0] > 0 and need == need[:1] * 3, (width, dtype, pre, need)


@pytest.mark.parametrize("dtype", [flare.FLARE_DT_BF16, flare.FLARE_DT_F32])
@pytest.mark.parametrize("pre", [0, 1])
def test_a_workspace_serves_smaller_batches(lib, pre, dtype):
    """More rows never need less, so that one workspace is sized by a program's largest batch."""
    counts = sorted({*range(0, 40), *range(40, 5000, 61), *(2 ** i + j for i in range(5, 31)
                                                          for j in (-1, 0, 1)), 2 ** 31 - 1})
    for width in (8, 64, 128, 512, 1024, 1368, 2048, 4096, 4104, 6016, 8192, 8200, 16384):
        last = 0
        for t in counts:
            need = flare.flare_block_norm_bwd_workspace_size(
                flare.block_norm_desc(t, width, dtype, pre_norm=pre))
            assert need >= last and need % (8 * width) == 0, (width, t)
            assert need > 0 or t == 0
            last = need
