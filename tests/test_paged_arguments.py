"""Tensors that the calls for ragged batches must not take for what they are not: other types, views with gaps, host memory."""
import re

import pytest
import torch

P = 1 << 20                                                           # an aligned address that no refused call touches


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


@pytest.fixture(autouse=True)
def no_device(k, monkeypatch):
    monkeypatch.setattr(k.binding.torch.cuda, "current_device", lambda: 0)


def _calls(k):
    """call -> (function, arguments by name, type wanted by name ("" any), names that are rows with a stride of the call)"""
    desc = k.make_paged_desc(8, 2, 128, 16, 4, 4)
    i32, f32, f16 = "torch.int32", "torch.float32", "torch.float16"
    plan = dict(desc=desc, base_len=P, new_len=P, n_requests=1, block_table=P, held_in=P, held_out=P, free_pages=P, free_count_in=P, free_count_out=P, max_rows=1,
                row_start=P, seq_len=P, slots=P, positions=P, refused=P)
    append = dict(desc=desc, qkv_dev=P, ld=1536, slots=P, positions=P, n_rows=1, rope_table=P, n_pos=64, q_out=P, ldq=1024, pages=P)
    read = dict(desc=desc, pages=P, slots=P, n_rows=1, kv_dev=P, ld=512)
    attention = dict(desc=desc, q_dev=P, q_type=k.KVPR_F16, ldq=1024, pages=P, block_table=P, row_start=P, seq_len=P, n_requests=1, n_rows=1, max_new=1, max_len=16, z_dev=P,
                     ldz=1024, ws_dev=P, ws_bytes=1 << 40)
    verify = dict(target_logits=P, draft_logits=P, logits_type=k.KVPR_F32, ld_target=100, ld_draft=100, vocab=100, tokens=P, row_start=P, n_requests=1, n_rows=1,
                  temperature=P, u_accept=P, u_sample=P, len_in=P, len_out=P, kept=P, out_tokens=P, ws_dev=P, ws_bytes=1 << 40)
    step = dict(verify, seq_len=P, certain=P)
    ints = lambda *names: {n: i32 for n in names}                                       # noqa: E731
    v = dict(ints("tokens", "row_start", "len_in", "len_out", "kept", "out_tokens"), temperature=f32, u_accept=f32, u_sample=f32, target_logits=f32, draft_logits=f32, ws_dev="")
    return {
        "plan": (k.kvpr_paged_plan, plan, ints(*(n for n, a in plan.items() if a == P)), ()),
        "append": (k.kvpr_paged_append, append, dict(ints("slots", "positions"), qkv_dev=f16, q_out=f16, rope_table=f32, pages=""), ("qkv_dev", "q_out")),
        "read": (k.kvpr_paged_read, read, dict(ints("slots"), kv_dev=f16, pages=""), ("kv_dev",)),
        "attention": (k.kvpr_paged_attention, attention, dict(ints("block_table", "row_start", "seq_len"), q_dev=f16, z_dev=f16, pages="", ws_dev=""), ("q_dev", "z_dev")),
        "verify": (k.kvpr_verify_drafts, verify, v, ("target_logits", "draft_logits")),
        "step": (k.kvpr_verify_step, step, dict(v, **ints("seq_len", "certain")), ("target_logits", "draft_logits")),
    }


NAMES = ("plan", "append", "read", "attention", "verify", "step")


@pytest.mark.parametrize("name", NAMES)
def test_every_array_is_listed(k, name):
    fn, args, types, _ = _calls(k)[name]
    assert {n for n, a in args.items() if a == P} == set(types)


@pytest.mark.parametrize("name", NAMES)
def test_other_types(k, name):
    fn, args, types, _ = _calls(k)[name]
    for at, want in types.items():
        for dtype in (torch.int64, torch.float64, torch.int32, torch.float32, torch.float16, torch.bfloat16):
            if want and str(dtype) != want:
                with pytest.raises(TypeError, match=re.escape(f"{at} must be {want}, got {dtype}")):
                    fn(**{**args, at: torch.zeros(16, dtype=dtype)}, stream=0)


@pytest.mark.parametrize("name", NAMES)
def test_views_with_gaps(k, name):
    fn, args, types, rows = _calls(k)[name]
    for at, want in types.items():
        dtype = getattr(torch, want[6:]) if want else torch.uint8
        wide = torch.zeros((4, 8), dtype=dtype)
        for view in (wide[:, ::2], wide[:, 1:3].t(), torch.zeros(16, dtype=dtype)[::2]):
            with pytest.raises(ValueError, match=f"the columns of {at} must lie" if at in rows else f"{at} must be contiguous"):
                fn(**{**args, at: view}, stream=0)
        # columns of a wider array: rows with a stride; a table or a pool cannot be that
        with pytest.raises(ValueError, match="current device" if at in rows else f"{at} must be contiguous"):
            fn(**{**args, at: wide[:, 2:6]}, stream=0)


@pytest.mark.parametrize("name", NAMES)
def test_host_memory_and_other_things(k, name):
    fn, args, types, _ = _calls(k)[name]
    for at, want in types.items():
        host = torch.zeros(16, dtype=getattr(torch, want[6:]) if want else torch.uint8)
        with pytest.raises(ValueError, match=f"{at} must be on the current device cuda:0, got cpu"):
            fn(**{**args, at: host}, stream=0)
        for other in (host.numpy(), [1, 2], 3.0, "x"):
            with pytest.raises(TypeError, match=f"{at} must be a tensor, an address or None"):
                fn(**{**args, at: other}, stream=0)


def test_a_type_argument_that_is_none_is_the_librarys_to_refuse(k):
    for name, arg, at in (("attention", "q_type", "q_dev"), ("verify", "logits_type", "target_logits"), ("step", "logits_type", "draft_logits")):
        fn, args, _, _ = _calls(k)[name]
        with pytest.raises(k.KvprError) as e:
            fn(**{**args, arg: 9}, stream=0)
        assert e.value.code == k.KVPR_E_INVAL
        with pytest.raises(ValueError, match="current device"):
            fn(**{**args, arg: 9, at: torch.zeros(16)}, stream=0)


def test_the_helper_itself(k):
    from paper_2411_17089_amd import _tensor_args as ta
    assert ta.addresses(0, "ib", ("a", "b"), None, 5) == [None, 5]
    assert ta.addresses(0, "", ()) == []
    for bad in ((), (0,), (0, "i"), (0, "i", ("a",)), (0, "i", ("a",), 1, 2), (0, "ii", ("a",), 1, 2), (0, 5, ("a",), 1), (0, "i", ["a"], 1), ("x", "i", ("a",), 1)):
        with pytest.raises(TypeError):
            ta.addresses(*bad)
    with pytest.raises((RuntimeError, ValueError)):
        ta.addresses(0, "b", ("a",), torch.zeros((3, 3)).to_sparse())


@pytest.mark.gpu
def test_addresses_on_the_gpu(k):
    from paper_2411_17089_amd import _tensor_args as ta
    t = [torch.zeros((3, 8), dtype=d, device="cuda") for d in (torch.int32, torch.float32, torch.float16, torch.float32, torch.uint8, torch.bfloat16)]
    d = t[0].device.index
    assert ta.addresses(d, "ifhsbr", tuple("abcdef"), *t) == [x.data_ptr() for x in t]
    views = [t[2][1:, 2:6], t[3][:, :3], t[5][::2]]
    assert ta.addresses(d, "hsr", tuple("abc"), *views) == [x.data_ptr() for x in views]
    with pytest.raises(ValueError, match="a must be contiguous"):
        ta.addresses(d, "i", ("a",), t[0][:, 1:])
    with pytest.raises(ValueError, match="must be on the current device cuda:%d" % (d + 1)):
        ta.addresses(d + 1, "i", ("a",), t[0])
