"""Speculative decoding, host side: refusals of the three entry points (all before any launch) and the plain forms against each other."""
import ctypes
import pathlib
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paper_2404_06910_b200 as sp
import spec_reference as ref
from workloads import build_layout

P = 1 << 20                    # an address that nothing is read from


def _tree_args(**change):
    lay = sp.binding._CLayout(1, 1, P, P, P, P, P, P, 10, 2, 8)
    a = dict(q=P, k_cache=P, v_cache=P, lay=ctypes.byref(lay), kept=P, k=1, tail_k=P, tail_v=P, tail_len=P, tail_cap=8, parent=P, n_nodes=None,
             max_nodes=4, max_keys=0, n_heads=4, n_kv_heads=2, head_dim=64, scale=1.0, out=P, lse=None, ws=P, ws_bytes=256, dtype=0, stream=None)
    a.update(change)
    return list(a.values()), lay


@pytest.mark.parametrize("change,code,text", [
    (dict(dtype=7), "INVALID_ARG", "dtype"), (dict(lay=None), "INVALID_ARG", "layout"), (dict(head_dim=96), "UNSUPPORTED", "head_dim"),
    (dict(n_kv_heads=3), "INVALID_ARG", "multiple"), (dict(n_kv_heads=0), "INVALID_ARG", "multiple"), (dict(k=4097), "INVALID_ARG", "k 4097"),
    (dict(k=-1), "INVALID_ARG", "k -1"), (dict(max_nodes=65), "UNSUPPORTED", "64"), (dict(max_nodes=-1), "INVALID_ARG", "negative"),
    (dict(tail_cap=-1), "INVALID_ARG", "negative"), (dict(max_keys=-1), "INVALID_ARG", "negative"), (dict(q=None), "INVALID_ARG", "NULL"),
    (dict(out=None), "INVALID_ARG", "NULL"), (dict(k_cache=None), "INVALID_ARG", "NULL"), (dict(kept=None), "INVALID_ARG", "kept_idx"),
    (dict(tail_k=None), "INVALID_ARG", "tail"), (dict(tail_len=None), "INVALID_ARG", "tail"), (dict(parent=None), "INVALID_ARG", "parent"),
    (dict(q=P + 8), "INVALID_ARG", "aligned"), (dict(tail_v=P + 4), "INVALID_ARG", "aligned"), (dict(ws=None), "WORKSPACE", "workspace"),
    (dict(ws=P + 16), "WORKSPACE", "workspace"), (dict(ws_bytes=255), "WORKSPACE", "workspace"),
    (dict(max_nodes=64, n_heads=2048, n_kv_heads=2048), "UNSUPPORTED", "65535"), (dict(tail_cap=2 ** 31 - 1), "UNSUPPORTED", "keys")])
def test_tree_refusals(change, code, text):
    args, _ = _tree_args(**change)
    assert sp.lib.sp_pruned_decode_tree(*args) == getattr(sp, "SP_ERR_" + code)
    assert text in sp.lib.sp_last_error().decode()


@pytest.mark.parametrize("dtype", [0, 1])
def test_tree_key_numbers_stay_below_2_31(dtype):
    """bf16 numbers keys from multiples of eight in every segment: up to seven numbers a segment that stand for no key count too.  (A path may be kept
    several times, so that this takes no 2^31 rows.)  The workspace is looked at behind the number of keys: without one nothing is launched."""
    k, pre, path = 4096, 2, 524272
    lay = sp.binding._CLayout(1, 1, P, P, P, P, P, P, 600000, pre, path)
    call = lambda cap: sp.lib.sp_pruned_decode_tree(*_tree_args(lay=ctypes.byref(lay), k=k, tail_cap=cap, ws=None, dtype=dtype)[0])
    most = 2 ** 31 - 1 - 256 - (pre + k * path) - (7 * (k + 1) if dtype else 0) - 1         # rows of the tail that are still fine
    assert call(most) == sp.SP_ERR_WORKSPACE
    assert call(most + 1) == sp.SP_ERR_UNSUPPORTED and "keys" in sp.lib.sp_last_error().decode()


def test_nothing_to_do_is_fine():
    assert sp.lib.sp_pruned_decode_tree(*_tree_args(max_nodes=0)[0]) == sp.SP_OK
    assert sp.lib.sp_sample_tokens(None, 8, 0, 8, None, None, None, None, None, None, None, 0, None) == sp.SP_OK
    assert sp.lib.sp_tree_accept(None, None, None, None, 0, 4, None, None, None, None, None, None, None, 0, 0, 0, 0, 0, 0, None) == sp.SP_OK


@pytest.mark.parametrize("change,code,text", [
    (dict(dtype=2), "INVALID_ARG", "dtype"), (dict(rows=-1), "INVALID_ARG", "n_rows"), (dict(vocab=0), "INVALID_ARG", "vocab"),
    (dict(ld=7), "INVALID_ARG", "ld_logits"), (dict(vocab=262145, ld=262145), "UNSUPPORTED", "vocab"), (dict(logits=None), "INVALID_ARG", "NULL"),
    (dict(u=None), "INVALID_ARG", "NULL"), (dict(tokens=None), "INVALID_ARG", "NULL"), (dict(logits=P + 2), "INVALID_ARG", "aligned"),
    (dict(rows=1 << 28), "UNSUPPORTED", "rows")])
def test_sample_refusals(change, code, text):
    a = dict(logits=P, ld=8, rows=2, vocab=8, u=P, temperature=None, top_k=None, top_p=None, min_p=None, tokens=P, logp=None, dtype=0, stream=None)
    a.update(change)
    assert sp.lib.sp_sample_tokens(*a.values()) == getattr(sp, "SP_ERR_" + code)
    assert text in sp.lib.sp_last_error().decode()


@pytest.mark.parametrize("change,code,text", [
    (dict(dtype=2), "INVALID_ARG", "dtype"), (dict(n_prompts=-1), "INVALID_ARG", "negative"), (dict(max_nodes=65), "UNSUPPORTED", "64"),
    (dict(n_accepted=None), "INVALID_ARG", "NULL"), (dict(draft=None), "INVALID_ARG", "NULL"), (dict(path=None), "INVALID_ARG", "NULL"),
    (dict(new_tail_len=None), "INVALID_ARG", "together"), (dict(tail_v=None), "INVALID_ARG", "tail"), (dict(tail_k=P + 8), "INVALID_ARG", "aligned"),
    (dict(ld_layer=8), "INVALID_ARG", "ld_layer"), (dict(head_dim=3, n_kv_heads=1), "UNSUPPORTED", "bytes"), (dict(n_kv_heads=0), "INVALID_ARG", "n_kv_heads"),
    (dict(new_tail_len=P + 4 * 4096 + 4), "INVALID_ARG", "overlap"), (dict(path=P + 16), "INVALID_ARG", "overlap"), (dict(n_prompts=65536), "UNSUPPORTED", "prompts")])
def test_accept_refusals(change, code, text):
    a = dict(draft=P, sampled=P + 4096, parent=P + 2 * 4096, n_nodes=P + 3 * 4096, n_prompts=2, max_nodes=4, path=2 * P, n_accepted=2 * P + 4096,
             next_token=2 * P + 8192, tail_k=4 * P, tail_v=5 * P, tail_len=P + 4 * 4096, new_tail_len=3 * P, tail_cap=8, n_layers=3, ld_layer=2 * 8 * 2 * 64,
             n_kv_heads=2, head_dim=64, dtype=0, stream=None)
    a.update(change)
    assert sp.lib.sp_tree_accept(*a.values()) == getattr(sp, "SP_ERR_" + code)
    assert text in sp.lib.sp_last_error().decode()


@pytest.mark.parametrize("k,v,text", [
    ((2, 2, 8, 2, 64), None, "come together"), (None, (2, 2, 8, 2, 64), "come together"),
    ((2, 1, 8, 2, 64), (2, 1, 8, 2, 64), "slots"), ((2, 2, 8, 2, 64), (2, 2, 7, 2, 64), "shape"), ((2, 2, 8, 2, 64), (1, 2, 8, 2, 64), "shape"),
    ((2, 2, 8, 2, 64), (2, 2, 8, 2, 128), "shape"), ((2, 2, 8, 2, 64), "bf16", "shape")])
def test_accept_takes_tails_alike_with_a_slot_for_every_prompt(k, v, text):
    """What the C entry point cannot see: refused before any launch."""
    make = lambda s, dtype=torch.float32: None if s is None else torch.zeros(s, dtype=dtype)
    tree, one = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match=text):
        sp.sp_tree_accept(tree, tree, tree, one, tree, one, one, make(k), make(k, torch.bfloat16) if v == "bf16" else make(v), one, one,
                          stream=SimpleNamespace(cuda_stream=0))


@pytest.mark.parametrize("layers,ld,away,apart", [
    (1, 0, 0, False), (1, 0, 4095, False), (1, 0, 4096, True), (1, 0, -4095, False), (1, 0, -4096, True),       # elements from the K to the V tail; a layer is 4096
    (3, 4096, 4096, False), (3, 4096, 2 * 4096, False), (3, 4096, 3 * 4096, True), (3, 4096, -2 * 4096, False), (3, 4096, -3 * 4096, True),
    (3, 8192, 4096, True), (3, 8192, 4092, False), (3, 8192, -4096, True), (3, 8192, -4100, False), (3, 10000, 4096, True), (3, 10000, 5904, True), (3, 10000, 5908, False),
    (3, 8192, 5 * 4096, True), (3, 8192, 4 * 4096, False), (3, 8192, 6 * 4096, True)])
def test_accept_refuses_k_and_v_tails_that_overlap(layers, ld, away, apart):
    """Two threads would move the same rows.  Tails that lie between one another (a layer's K, its V, the next layer's K) are fine: they get as far as
    the check of the outputs, which overlap an input here, so that nothing is launched."""
    at, away = 16 * P, away // 4 * 4 if away >= 0 else -(-away // 4 * 4)
    code = sp.lib.sp_tree_accept(P, P + 4096, P + 2 * 4096, None, 2, 4, P + 16, 2 * P, 3 * P, at, at + 4 * away, P + 4 * 4096, 4 * P, 16, layers, ld, 2, 64, 0, None)
    assert code == sp.SP_ERR_INVALID_ARG
    assert ("outputs" if apart else "tails overlap") in sp.lib.sp_last_error().decode()


def _call_with(name, **types):
    """A call of the front end that has nothing to do, with tensors of the given types in place of int32 and fp32."""
    i32 = lambda n, *s: torch.zeros(s, dtype=types.get(n, torch.int32))
    f32 = lambda n, *s: torch.zeros(s, dtype=types.get(n, torch.float32))
    stream = SimpleNamespace(cuda_stream=0)
    if name == "tree":
        x, lay = torch.zeros(1, 0, 4, 64), sp.DeviceLayout.from_host(build_layout([2], [[2]], [[1]]), "cpu")
        tail = torch.zeros(1, 4, 4, 64)
        sp.sp_pruned_decode_tree(x, tail[0], tail[0], lay, i32("kept_idx", 1, 1), 1, tail, tail, i32("tail_len", 1), 4, i32("parent", 1, 0), i32("n_nodes", 1), 0.1, x, f32("lse", 1, 0, 4),
                                 torch.zeros(256, dtype=torch.uint8), stream=stream)
    elif name == "sample":
        sp.sp_sample_tokens(torch.zeros(0, 8), f32("u", 0), i32("tokens", 0), f32("logp", 0), temperature=f32("temperature", 0), top_k=i32("top_k", 0), top_p=f32("top_p", 0),
                            min_p=f32("min_p", 0), stream=stream)
    else:
        tree = lambda n: i32(n, 0, 4)
        sp.sp_tree_accept(tree("draft"), tree("sampled"), tree("parent"), i32("n_nodes", 0), tree("path"), i32("n_accepted", 0), i32("next_token", 0), torch.zeros(1, 0, 8, 2, 64),
                          torch.zeros(1, 0, 8, 2, 64), i32("tail_len", 0), i32("new_tail_len", 0), stream=stream)


@pytest.mark.parametrize("name,arguments", [
    ("tree", ["kept_idx", "tail_len", "parent", "n_nodes", "lse"]), ("sample", ["u", "tokens", "logp", "temperature", "top_k", "top_p", "min_p"]),
    ("accept", ["draft", "sampled", "parent", "n_nodes", "path", "n_accepted", "next_token", "tail_len", "new_tail_len"])])
def test_tensors_of_other_types_are_refused(name, arguments):
    """Whole numbers are int64 and reals fp32 or fp64 where nobody says otherwise: not to be read as if they were int32 and fp32."""
    _call_with(name)
    for a in arguments:
        for wrong in (torch.int64, torch.float64, torch.float32 if a not in ("u", "logp", "lse", "temperature", "top_p", "min_p") else torch.int32):
            with pytest.raises(TypeError, match="int32|float32"):
                _call_with(name, **{a: wrong})


def test_no_kernel_waits_for_the_lanes_that_happen_to_be_there():
    """A barrier over __activemask() orders nothing that the compiler did not keep together by itself; that it did so cannot be tested by running."""
    csrc = pathlib.Path(sp.binding.LIB_PATH).parent / "csrc"
    assert not [f.name for f in csrc.iterdir() if f.suffix in (".cu", ".cuh") and "__activemask" in f.read_text()]


def test_plain_tree_of_a_chain_is_causal_attention():
    """In the plain form a chain behind a context is causal attention over the concatenation."""
    rng = np.random.default_rng(0)
    lay = build_layout([3], [[4, 2]], [[2, 1]])
    N, H, D, t = 4, 2, 8, 2
    q, kc, vc = rng.normal(size=(1, N, H, D)), rng.normal(size=(lay.total_tokens, H, D)), rng.normal(size=(lay.total_tokens, H, D))
    tk, tv = rng.normal(size=(1, 8, H, D)), rng.normal(size=(1, 8, H, D))
    out, lse, _, _ = ref.tree_attention(q, kc, vc, lay, np.array([[1, 0]]), tk, tv, [t], np.array([[-1, 0, 1, 2]]), [N], 0.3)
    rows = [0, 1, 2, *range(9, 12), *range(3, 9)]
    for i in range(N):
        k, v = np.concatenate([kc[rows], tk[0, :t + i + 1]]), np.concatenate([vc[rows], tv[0, :t + i + 1]])
        s = 0.3 * np.einsum("hd,khd->hk", q[0, i], k)
        p = np.exp(s) / np.exp(s).sum(1, keepdims=True)
        np.testing.assert_allclose(out[0, i], np.einsum("hk,khd->hd", p, v), rtol=1e-12)
        np.testing.assert_allclose(lse[0, i], np.log(np.exp(s).sum(1)), rtol=1e-12)


def test_plain_sampling_by_hand():
    x = np.log(np.array([[0.1, 0.4, 0.1, 0.4]]))
    take = lambda u, **f: int(ref.sample(x, [u], **f)[0][0])
    assert [take(u) for u in (0.0, 0.05, 0.11, 0.49, 0.51, 0.59, 0.61, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [take(u, top_k=[2]) for u in (0.0, 0.49, 0.51)] == [1, 1, 3]
    assert [take(u, top_k=[3]) for u in (0.0, 0.2)] == [0, 1]              # of the two equal ones the first stays
    assert [take(u, top_p=[0.4]) for u in (0.0, 0.9)] == [1, 1] and [take(u, top_p=[0.5]) for u in (0.0, 0.9)] == [1, 3]
    assert [take(u, min_p=[0.5]) for u in (0.0, 0.9)] == [1, 3] and take(0.9, temperature=[0.0]) == 1
