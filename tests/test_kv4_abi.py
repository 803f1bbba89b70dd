"""Host-side refusals of the calls on the 4-bit cache (no GPU: the checks fail before anything is enqueued)."""
import ctypes

import pytest
import torch

from paper_2607_11976_b200 import binding, build

FAKE, ODD, NULL = 0x1000, 0x1004, None
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3
BF16, F32, E4M3 = 1, 0, 2


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def test_page_bytes(lib):
    assert lib.lt_kv4_page_bytes(8, 128) == 8 * 64 * 144 and lib.lt_kv4_page_bytes(1, 64) == 64 * 72
    assert lib.lt_kv4_page_bytes(0, 128) == lib.lt_kv4_page_bytes(8, 96) == lib.lt_kv4_page_bytes(2000, 64) == 0
    assert lib.lt_kv4_attention_workspace_bytes(BF16, 4, 2, 16, 8, 128) > 0
    assert lib.lt_kv4_attention_workspace_bytes(BF16, 4, 2, 12, 8, 128) == 0
    assert lib.lt_kv4_attention_workspace_bytes(E4M3, 4, 2, 16, 8, 128) == 0


TABLES = dict(context_len=FAKE, new_len=FAKE, free_pages=FAKE, n_free=4, B=2, max_pages=8, T=16, page_table=FAKE, total_len=0x2000,
              query_start=FAKE, slot_map=FAKE, position=FAKE, status=FAKE, stream=NULL)


@pytest.mark.parametrize("change", [dict(context_len=NULL), dict(new_len=NULL), dict(free_pages=NULL), dict(n_free=-1), dict(B=0),
                                    dict(B=(1 << 20) + 1), dict(max_pages=0), dict(max_pages=(1 << 24) + 1), dict(T=0), dict(T=(1 << 24) + 1), dict(page_table=NULL), dict(total_len=NULL),
                                    dict(total_len=FAKE), dict(query_start=NULL), dict(slot_map=NULL), dict(position=NULL),
                                    dict(status=NULL)], ids=str)
def test_page_tables_refuses(lib, change):
    assert lib.lt_page_tables(*{**TABLES, **change}.values()) == INVALID


APPEND = dict(dtype=BF16, k=FAKE, v=FAKE, k_stride=1024, v_stride=1024, slot_map=FAKE, T=4, Hkv=8, D=128, pool=FAKE, pages=10, stream=NULL)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=E4M3), UNSUPPORTED), (dict(dtype=7), UNSUPPORTED), (dict(D=96), UNSUPPORTED), (dict(D=256), UNSUPPORTED),
    (dict(Hkv=1025), UNSUPPORTED), (dict(Hkv=0), INVALID), (dict(k=NULL), INVALID), (dict(v=NULL), INVALID), (dict(k=ODD), INVALID),
    (dict(v=ODD), INVALID), (dict(k_stride=1016), INVALID), (dict(v_stride=1028), INVALID), (dict(k_stride=-2048), INVALID),
    (dict(slot_map=NULL), INVALID), (dict(T=0), INVALID), (dict(pool=NULL), INVALID), (dict(pool=ODD), INVALID), (dict(pages=0), INVALID),
    (dict(pages=1 << 25), INVALID), (dict(dtype=F32, k_stride=1026), INVALID)], ids=str)
def test_append_refuses(lib, change, code):
    assert lib.lt_kv4_append(*{**APPEND, **change}.values()) == code


READ = dict(dtype=BF16, pool=FAKE, pages=10, slots=FAKE, n=4, Hkv=8, D=128, k_out=FAKE, v_out=FAKE, stream=NULL)


@pytest.mark.parametrize("change,code", [
    (dict(dtype=E4M3), UNSUPPORTED), (dict(D=32), UNSUPPORTED), (dict(pool=NULL), INVALID), (dict(pages=-1), INVALID), (dict(slots=NULL), INVALID),
    (dict(n=0), INVALID), (dict(Hkv=-1), INVALID), (dict(k_out=NULL), INVALID), (dict(v_out=ODD), INVALID)], ids=str)
def test_read_refuses(lib, change, code):
    assert lib.lt_kv4_read(*{**READ, **change}.values()) == code


ATTN = dict(dtype=BF16, q=FAKE, q_stride=2048, pool=FAKE, pages=10, page_table=FAKE, max_pages=4, query_start=FAKE, context_len=FAKE, B=2, T=4,
            Hq=16, Hkv=8, D=128, max_new=0, scale=0.1, out=FAKE, lse=NULL, workspace=FAKE, bytes=1 << 32, tunables=None, stream=NULL)
REFUSED = [
    (dict(dtype=E4M3), UNSUPPORTED), (dict(D=192), UNSUPPORTED), (dict(q=NULL), INVALID), (dict(q=ODD), INVALID), (dict(q_stride=2040), INVALID),
    (dict(q_stride=2052), INVALID), (dict(pool=NULL), INVALID), (dict(pages=0), INVALID), (dict(page_table=NULL), INVALID),
    (dict(max_pages=0), INVALID), (dict(query_start=NULL), INVALID), (dict(context_len=NULL), INVALID), (dict(B=0), INVALID),
    (dict(T=0), INVALID), (dict(T=(1 << 24) + 1), INVALID), (dict(B=(1 << 20) + 1), INVALID), (dict(max_pages=(1 << 24) + 1), INVALID),
    (dict(T=1 << 20, Hq=1 << 15, q_stride=1 << 22), INVALID), (dict(Hq=12), INVALID), (dict(Hq=0), INVALID), (dict(Hkv=0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(out=NULL), INVALID), (dict(out=ODD), INVALID), (dict(workspace=NULL), WORKSPACE),
    (dict(workspace=0x1010), WORKSPACE), (dict(bytes=16), WORKSPACE),
    (dict(tunables=binding.Tunables(path=binding.LT_PATH_FUSED_ABS)), INVALID), (dict(tunables=binding.Tunables(path=9)), INVALID),
    (dict(dtype=F32, tunables=binding.Tunables(path=binding.LT_PATH_FUSED)), UNSUPPORTED)]


@pytest.mark.parametrize("change,code", REFUSED + [(dict(max_new=-1), INVALID)], ids=str)
def test_attention_refuses(lib, change, code):
    a = {**ATTN, **change}
    a["tunables"] = None if a["tunables"] is None else ctypes.byref(a["tunables"])
    assert lib.lt_kv4_attention(*a.values()) == code


@pytest.mark.parametrize("change,code", REFUSED + [(dict(idx=NULL), INVALID), (dict(topk=0), INVALID), (dict(topk=8193), INVALID)], ids=str)
def test_attention_topk_refuses(lib, change, code):
    a = {}
    for name, value in ATTN.items():
        if name != "max_new":
            a[name] = value
        if name == "context_len":
            a["idx"], a["topk"] = FAKE, 64
    a.update(change)
    a["tunables"] = None if a["tunables"] is None else ctypes.byref(a["tunables"])
    assert lib.lt_kv4_attention_topk(*a.values()) == code


def test_binding_refuses_tensors_that_do_not_fit():
    pool = torch.zeros(3, 2, 64, 144, dtype=torch.uint8)
    x = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    i = torch.zeros(4, dtype=torch.int32)
    for bad in (torch.zeros(3, 2, 64, 145, dtype=torch.uint8), torch.zeros(3, 2, 32, 144, dtype=torch.uint8), pool.int(), pool[0]):
        with pytest.raises(ValueError):
            binding.lt_kv4_append("bf16", x, x, i, bad)
    with pytest.raises(ValueError):
        binding.lt_kv4_append("bf16", x, x[:, :1], i, pool)
    with pytest.raises(ValueError):
        binding.lt_kv4_append("bf16", x, x, i.long(), pool)
    with pytest.raises(ValueError):
        binding.lt_kv4_append("bf16", x, x, i, pool)  # not on a GPU
    with pytest.raises(ValueError):
        binding.lt_kv4_read("f32", pool, i, x, x)
    with pytest.raises(ValueError):
        binding.lt_page_tables(i, i[:3], i, torch.zeros(4, 2, dtype=torch.int32), i, i, i, i, i)
    with pytest.raises(ValueError):
        binding.alloc_kv4_pool(4, 8, 96, device="cpu")
    assert binding.alloc_kv4_pool(4, 8, 64, device="cpu").shape == (4, 8, 64, 72)
