"""CPU checks of the tree calls' host side: every refusal happens before any CUDA
work.  The pointers are stand-ins on the right boundaries; no call gets past
its checks, except those on zero requests, which launch nothing."""
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


def softmax(**kw):
    d = flare.softmax_desc(2, 16, 16, 2, 256, 64, 100, 64, flare.FLARE_DT_BF16, 0.0625)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def linear(**kw):
    d = flare.linear_desc(2, 16, 16, 32, 128, 128, 6, flare.FLARE_DT_BF16, 0.088)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def verify(**kw):
    d = flare.tree_verify_desc(2, 16, 1000, flare.FLARE_DT_BF16)
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def layers(n, at=AT):
    return (ctypes.c_void_p * max(n, 1))(*[at] * n)


def arguments(call, desc=None, n_layers=2):
    """[name, value] of a call that all host checks accept."""
    size = ctypes.c_size_t(0)
    if call == "flare_tree_softmax_attn":
        d = softmax() if desc is None else desc
        flare.load().flare_tree_softmax_workspace_size(ctypes.byref(d), ctypes.byref(size))
        names = ("q k_blk v_blk k_pool v_pool page_table prefix_len parent node_len out lse "
                 "workspace").split()
        return [["desc", ctypes.byref(d)]] + [[n, AT] for n in names] + \
            [["workspace_bytes", size.value], ["dev_status", AT], ["stream", None]]
    if call == "flare_tree_linear_attn":
        d = linear() if desc is None else desc
        names = ("q k v log_decay beta state_pool state_slot parent node_len out "
                 "dev_status").split()
        return [["desc", ctypes.byref(d)]] + [[n, AT] for n in names] + [["stream", None]]
    if call == "flare_tree_verify":
        d = verify() if desc is None else desc
        flare.load().flare_tree_verify_workspace_size(ctypes.byref(d), ctypes.byref(size))
        names = ("logits draft_probs token parent node_len uniform noise path path_len next_token "
                 "node_logp workspace").split()
        return [["desc", ctypes.byref(d)]] + [[n, AT] for n in names] + \
            [["workspace_bytes", size.value], ["dev_status", AT], ["stream", None]]
    if call == "flare_tree_commit_state":
        d = linear() if desc is None else desc
        names = ("k v log_decay beta state_pool src_slot dst_slot path path_len "
                 "dev_status").split()
        return [["desc", ctypes.byref(d)]] + [[n, AT] for n in names] + [["stream", None]]
    d = softmax() if desc is None else desc
    return [["desc", ctypes.byref(d)], ["num_layers", n_layers]] + \
        [[n, layers(n_layers)] for n in ("k_blk", "v_blk", "k_pool", "v_pool")] + \
        [[n, AT] for n in ("page_table", "prefix_len", "path", "path_len", "dev_status")] + \
        [["stream", None]]


def run(lib, call, args, **change):
    names = [n for n, _ in args]
    assert all(k in names for k in change)
    return getattr(lib, call)(*[change.get(n, v) for n, v in args])


CALLS = ("flare_tree_softmax_attn", "flare_tree_linear_attn", "flare_tree_verify",
         "flare_tree_commit_state", "flare_tree_append_kv")
MAY_BE_NULL = {"stream", "lse", "draft_probs"}


@pytest.mark.parametrize("call", CALLS)
def test_every_pointer_is_needed(lib, call):
    args = arguments(call)
    for name, value in args:
        if name in MAY_BE_NULL or name in ("workspace_bytes", "num_layers"):
            continue
        assert run(lib, call, args, **{name: None}) == BAD, name


@pytest.mark.parametrize("call,names", [
    ("flare_tree_softmax_attn", "q k_blk v_blk k_pool v_pool out"),
    ("flare_tree_linear_attn", "q k v state_pool out"),
    ("flare_tree_commit_state", "k v state_pool")])
def test_vector_operands_start_on_16_bytes(lib, call, names):
    args = arguments(call)
    for name in names.split():
        assert run(lib, call, args, **{name: AT + 8}) == BAD, name


def test_verify_operands_start_on_their_elements(lib):
    args = arguments("flare_tree_verify")
    for name, off in (("logits", 1), ("draft_probs", 2), ("noise", 2)):
        assert run(lib, "flare_tree_verify", args, **{name: AT + off}) == BAD, name
    args = arguments("flare_tree_verify", verify(logits_dtype=flare.FLARE_DT_F32))
    assert run(lib, "flare_tree_verify", args, logits=AT + 2) == BAD


@pytest.mark.parametrize("call", ["flare_tree_softmax_attn", "flare_tree_verify"])
def test_workspace_size_and_boundary(lib, call):
    args = arguments(call)
    size = dict((n, v) for n, v in args)["workspace_bytes"]
    assert size > 0
    assert run(lib, call, args, workspace_bytes=size - 1) == BAD
    assert run(lib, call, args, workspace=AT + 128) == BAD


@pytest.mark.parametrize("call,make", [
    ("flare_tree_softmax_attn", softmax), ("flare_tree_append_kv", softmax),
    ("flare_tree_linear_attn", linear), ("flare_tree_commit_state", linear)])
def test_shapes_of_the_two_layer_kinds(lib, call, make):
    cases = [(dict(num_requests=-1), BAD), (dict(block_len=0), BAD), (dict(block_len=65), NO),
             (dict(act_dtype=7), BAD)]
    if make is softmax:
        cases += [(dict(num_q_heads=15), BAD), (dict(head_dim=96), NO), (dict(page_size=48), NO)]
    else:
        cases += [(dict(num_v_heads=24), BAD), (dict(head_dim_k=96), NO),
                  (dict(head_dim_v=256), NO)]
    for change, want in cases:
        args = arguments(call, make(**change))
        assert run(lib, call, args) == want, change


def test_the_softmax_calls_ignore_mask_fields(lib):
    n, m = ctypes.c_size_t(0), ctypes.c_size_t(0)
    d = softmax(mask_mode=7)
    assert lib.flare_tree_softmax_workspace_size(ctypes.byref(d), ctypes.byref(n)) == OK
    assert lib.flare_tree_softmax_workspace_size(ctypes.byref(softmax()), ctypes.byref(m)) == OK
    assert n.value == m.value and n.value % 256 == 0
    assert lib.flare_tree_softmax_workspace_size(ctypes.byref(d), None) == BAD


def test_verify_descriptor(lib):
    n = ctypes.c_size_t(0)
    inf, nan = float("inf"), float("nan")
    for change, want in [
            (dict(num_requests=-1), BAD), (dict(num_nodes=0), BAD), (dict(num_nodes=65), NO),
            (dict(vocab_size=0), BAD), (dict(vocab_size=(1 << 24) + 1), NO),
            (dict(logits_dtype=9), BAD), (dict(mode=2), BAD), (dict(inv_temperature=0.0), BAD),
            (dict(inv_temperature=-1.0), BAD), (dict(inv_temperature=inf), BAD),
            (dict(inv_temperature=nan), BAD)]:
        d = verify(**change)
        assert lib.flare_tree_verify_workspace_size(ctypes.byref(d), ctypes.byref(n)) == want, change
        assert run(lib, "flare_tree_verify", arguments("flare_tree_verify", d)) == want, change
    d = verify(mode=flare.FLARE_VERIFY_GREEDY, inv_temperature=0.0)  # not read
    assert lib.flare_tree_verify_workspace_size(ctypes.byref(d), ctypes.byref(n)) == OK
    assert lib.flare_tree_verify_workspace_size(ctypes.byref(d), None) == BAD


def test_append_layers(lib):
    call = "flare_tree_append_kv"
    assert run(lib, call, arguments(call, n_layers=0)) == BAD
    assert run(lib, call, arguments(call, n_layers=65)) == NO
    args = arguments(call)
    for name in ("k_blk", "v_blk", "k_pool", "v_pool"):
        for bad in (None, AT + 8):
            assert run(lib, call, args, **{name: (ctypes.c_void_p * 2)(AT, bad)}) == BAD, name


@pytest.mark.parametrize("call,make", list(zip(CALLS, (softmax, linear, verify, linear,
                                                        softmax))))
def test_no_requests_is_no_work(lib, call, make):
    before = lib.flare_launch_count()
    assert run(lib, call, arguments(call, make(num_requests=0))) == OK
    assert lib.flare_launch_count() == before


def test_binding_refuses_strided_tensors_and_uneven_layer_lists(lib):
    t = torch.zeros(4, 4)
    with pytest.raises(ValueError, match="contiguous"):
        flare.flare_tree_commit_state(linear(), t.t()[1:], *[t] * 10)
    with pytest.raises(ValueError, match="per layer"):
        flare.flare_tree_append_kv(softmax(), [t], [t, t], [t], [t], t, t, t, t, t)
    with pytest.raises(flare.FlareError):
        flare.flare_tree_softmax_workspace_size(softmax(head_dim=80))
    with pytest.raises(flare.FlareError):
        flare.flare_tree_verify_workspace_size(verify(vocab_size=0))
