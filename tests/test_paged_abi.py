"""What the entry points for ragged batches refuse, before anything touches the GPU."""
import pytest


@pytest.fixture(scope="module")
def k():
    import paper_2411_17089_amd as k
    return k


GOOD = dict(n_heads=8, n_kv_heads=2, head_dim=128, page_size=16, n_pages=4, table_width=4)
BAD = [(dict(head_dim=96), "E_INVAL"), (dict(n_heads=0), "E_RANGE"), (dict(n_heads=70000, n_kv_heads=70000), "E_RANGE"), (dict(n_heads=16385, n_kv_heads=1), "E_RANGE"), (dict(n_kv_heads=0), "E_RANGE"),
       (dict(n_kv_heads=3), "E_INVAL"), (dict(page_size=8), "E_INVAL"), (dict(page_size=48), "E_INVAL"), (dict(page_size=512), "E_INVAL"),
       (dict(n_pages=0), "E_RANGE"), (dict(n_pages=1 << 27), "E_RANGE"), (dict(table_width=0), "E_RANGE"), (dict(table_width=1 << 27), "E_RANGE")]


def _calls(k, desc):
    P = 1 << 20                                                       # an aligned address that no refused call touches
    return {
        "plan": (k.kvpr_paged_plan, [desc, P, P, 1, P, P, P, P, P, P, 1, P, P, P, P, P]),
        "append": (k.kvpr_paged_append, [desc, P, 1536, P, P, 1, P, 64, P, 1024, P]),
        "read": (k.kvpr_paged_read, [desc, P, P, 1, P, 512]),
        "attention": (k.kvpr_paged_attention, [desc, P, k.KVPR_F16, 1024, P, P, P, P, 1, 1, 1, 16, P, 1024, P, 1 << 40]),
        "verify": (k.kvpr_verify_drafts, [P, P, k.KVPR_F32, 100, 100, 100, P, P, 1, 1, P, P, P, P, P, P, P, P, 1 << 40]),
    }


@pytest.fixture(autouse=True)
def no_device(k, monkeypatch):
    monkeypatch.setattr(k.binding.torch.cuda, "current_device", lambda: 0)


@pytest.mark.parametrize("change,code", BAD)
def test_bad_descriptions(k, change, code):
    desc = k.make_paged_desc(**{**GOOD, **change})
    assert k.kvpr_page_bytes(desc) == 0
    assert k.kvpr_paged_attention_workspace_bytes(desc, 1, 1, 1, 1) == 0
    for name, (fn, args) in _calls(k, desc).items():
        if name == "verify":
            continue
        with pytest.raises(k.KvprError) as e:
            fn(*args, stream=0)
        assert e.value.code == getattr(k, "KVPR_" + code), name


# call, argument, value, code
ARGS = [("plan", 3, 0, "E_RANGE"), ("plan", 3, 8193, "E_RANGE"), ("plan", 10, -1, "E_RANGE"), ("plan", 10, (1 << 30) + 1, "E_RANGE"), ("append", 5, (1 << 30) + 1, "E_RANGE"),
        ("read", 3, (1 << 30) + 1, "E_RANGE"), ("attention", 9, (1 << 28) + 1, "E_RANGE"), ("verify", 9, 1 << 23, "E_RANGE")] + \
       [("plan", i, None, "E_INVAL") for i in (1, 2, 4, 5, 6, 7, 8, 9, 11, 12, 13, 14, 15)] + \
       [("append", 2, 1528, "E_INVAL"), ("append", 2, 1540, "E_INVAL"), ("append", 5, -1, "E_RANGE"), ("append", 7, 0, "E_RANGE"), ("append", 6, None, "E_INVAL"),
        ("append", 9, 1016, "E_INVAL"), ("append", 9, 1028, "E_INVAL"), ("append", 1, (1 << 20) + 8, "E_INVAL"), ("append", 8, (1 << 20) + 2, "E_INVAL"),
        ("append", 10, (1 << 20) + 4, "E_INVAL")] + [("append", i, None, "E_INVAL") for i in (1, 3, 4, 10)] + \
       [("read", 3, -1, "E_RANGE"), ("read", 5, 504, "E_INVAL"), ("read", 5, 514, "E_INVAL"), ("read", 4, (1 << 20) + 2, "E_INVAL")] + \
       [("read", i, None, "E_INVAL") for i in (1, 2, 4)] + \
       [("attention", 2, 3, "E_INVAL"), ("attention", 3, 1016, "E_INVAL"), ("attention", 3, 1028, "E_INVAL"), ("attention", 8, 0, "E_RANGE"),
        ("attention", 8, 8193, "E_RANGE"), ("attention", 9, -1, "E_RANGE"), ("attention", 10, 0, "E_RANGE"), ("attention", 11, 0, "E_RANGE"),
        ("attention", 13, 1020, "E_INVAL"), ("attention", 1, (1 << 20) + 8, "E_INVAL"), ("attention", 12, (1 << 20) + 2, "E_INVAL"), ("attention", 15, 0, "E_INVAL"),
        ("attention", 14, (1 << 20) + 8, "E_INVAL")] + [("attention", i, None, "E_INVAL") for i in (1, 4, 5, 6, 7, 12, 14)] + \
       [("verify", 2, 7, "E_INVAL"), ("verify", 3, 99, "E_INVAL"), ("verify", 4, 99, "E_INVAL"), ("verify", 5, 0, "E_RANGE"), ("verify", 5, (1 << 24) + 1, "E_RANGE"),
        ("verify", 8, 0, "E_RANGE"), ("verify", 9, -1, "E_RANGE"), ("verify", 13, None, "E_INVAL"), ("verify", 14, None, "E_INVAL"), ("verify", 18, 0, "E_INVAL"),
        ("verify", 0, (1 << 20) + 2, "E_INVAL"), ("verify", 17, (1 << 20) + 8, "E_INVAL")] + [("verify", i, None, "E_INVAL") for i in (0, 6, 7, 10, 11, 12, 15, 16, 17)]


@pytest.mark.parametrize("name,at,value,code", ARGS)
def test_bad_arguments(k, name, at, value, code):
    fn, args = _calls(k, k.make_paged_desc(**GOOD))[name]
    args[at] = value
    with pytest.raises(k.KvprError) as e:
        fn(*args, stream=0)
    assert e.value.code == getattr(k, "KVPR_" + code)
    assert k.kvpr_last_error()


def test_null_description_and_sizes(k):
    assert k.lib.kvpr_paged_read(None, 1 << 20, 1 << 20, 1, 1 << 20, 512, None) == k.KVPR_E_INVAL
    desc = k.make_paged_desc(**GOOD)
    assert k.kvpr_page_bytes(desc) == 16 * 2 * 144
    assert k.kvpr_page_bytes(k.make_paged_desc(**{**GOOD, "head_dim": 64, "page_size": 256})) == 256 * 2 * 72
    for bad in ((0, 1, 1, 1), (8193, 1, 1, 1), (1, -1, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0)):
        assert k.kvpr_paged_attention_workspace_bytes(desc, *bad) == 0
    assert k.kvpr_paged_attention_workspace_bytes(desc, 8192, 1 << 20, 1 << 20, 1 << 30) > 0
    assert k.kvpr_verify_workspace_bytes(0, 1, 100) == 0 and k.kvpr_verify_workspace_bytes(1, 1, 0) == 0 and k.kvpr_verify_workspace_bytes(1, 0, 1) > 0


def test_append_without_rotation_wants_no_q_out(k):
    fn, args = _calls(k, k.make_paged_desc(**GOOD))["append"]
    args[6], args[4] = None, None
    with pytest.raises(k.KvprError) as e:
        fn(*args, stream=0)
    assert e.value.code == k.KVPR_E_INVAL and "q_out" in str(e.value)


def test_nothing_to_do_is_no_error(k):
    desc = k.make_paged_desc(**GOOD)
    calls = _calls(k, desc)
    for name, rows, nulls in (("append", 5, (1, 3, 4, 10)), ("read", 3, (1, 2, 4)), ("attention", 9, (1, 4, 5, 6, 7, 12))):
        fn, args = calls[name]
        args[rows] = 0
        for i in nulls:
            args[i] = None
        fn(*args, stream=0)


def test_tensors_of_the_wrong_kind(k):
    import torch
    desc = k.make_paged_desc(**GOOD)
    host = torch.zeros(16, dtype=torch.int32)
    for name, at in (("plan", 1), ("append", 3), ("read", 2), ("attention", 5), ("verify", 6)):
        fn, args = _calls(k, desc)[name]
        args[at] = host
        with pytest.raises(ValueError, match="current device"):
            fn(*args, stream=0)
    for name, at in (("append", 1), ("append", 8), ("append", 6), ("read", 4), ("attention", 1), ("attention", 12), ("verify", 0), ("verify", 1)):
        fn, args = _calls(k, desc)[name]
        args[at] = torch.zeros(16, dtype=torch.int32)
        with pytest.raises(TypeError, match="must be torch.float"):
            fn(*args, stream=0)
