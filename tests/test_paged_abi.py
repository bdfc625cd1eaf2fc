"""What the kvev_paged_* entry points refuse, before any device work (no GPU needed)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def kv():
    from paper_2606_15157_gb300 import build, kvev
    build.build()
    kvev.load()
    return kvev


P = 1 << 20  # stands for a device pointer: 16-byte aligned, never read by the host


def desc(kv, **kw):
    a = {"K": P, "V": P, "page_stride": 16 * 8 * 128, "token_stride": 8 * 128, "head_stride": 128, "num_pages": 64,
         "page_size": 16, "H_kv": 8, "d": 128, "dtype": kv.BF16, **kw}
    d = kv.PagedCacheDesc(*[a[n] for n, _ in kv.PagedCacheDesc._fields_])
    return d


BAD_CACHES = [({"K": 0}, "EINVAL"), ({"V": 0}, "EINVAL"), ({"K": P + 8}, "EINVAL"), ({"V": P + 2}, "EINVAL"), ({"page_stride": 0}, "EINVAL"),
              ({"token_stride": -1024}, "EINVAL"), ({"head_stride": 132}, "EINVAL"), ({"num_pages": 0}, "EINVAL"), ({"page_size": 0}, "EINVAL"),
              ({"page_size": 24}, "EINVAL"), ({"page_size": 4}, "EINVAL"), ({"page_size": 512}, "EINVAL"), ({"num_pages": 1 << 27}, "EINVAL"),
              ({"H_kv": 0}, "EINVAL"), ({"d": 96}, "ENOTSUP"), ({"d": 0}, "ENOTSUP"), ({"dtype": 2}, "EINVAL")]


def calls(kv):
    """name -> (function, good keyword arguments)"""
    cache = desc(kv)
    at = C.addressof(cache)
    need = kv.kvev_paged_attention_workspace(32, 8, 128)
    return cache, {
        "tables": (kv.kvev_paged_tables, dict(lens=P, new_lens=P, B=4, page_size=16, num_pages=64, free_pages=P, free_count=P, block_table=P,
                                              max_pages=8, T=9, kv_lens=P, cu_new=P, slots=P, positions=P, granted=P, free_count_out=P,
                                              device_status=P, stream=None)),
        "release": (kv.kvev_paged_release, dict(lens=P, done=P, B=4, page_size=16, num_pages=64, block_table=P, max_pages=8, free_pages=P,
                                                free_count=P, lens_out=P, free_count_out=P, device_status=P, stream=None)),
        "write": (kv.kvev_paged_write, dict(cache=at, k=P, v=P, token_stride=1024, head_stride=128, slots=P, T=9, device_status=P, stream=None)),
        "gather": (kv.kvev_paged_gather, dict(cache=at, block_table=P, max_pages=8, lens=P, B=4, S_cap=128, out_K=P, out_V=P,
                                              device_status=P, stream=None)),
        "attention": (kv.kvev_paged_attention, dict(cache=at, q=P, q_token_stride=4096, q_head_stride=128, cu_new=P, kv_lens=P, block_table=P,
                                                    max_pages=8, B=4, T=9, H_q=32, scale=0.0, window=0, out=P, out_token_stride=4096,
                                                    out_head_stride=128, lse=P, workspace=P, workspace_bytes=need, device_status=P,
                                                    stream=None))}


BAD_ARGS = [("tables", {k: 0}, "EINVAL") for k in ("lens", "new_lens", "free_pages", "free_count", "block_table", "kv_lens", "cu_new", "slots",
                                                   "positions", "granted", "free_count_out", "device_status")]
BAD_ARGS += [("release", {k: 0}, "EINVAL") for k in ("lens", "done", "block_table", "free_pages", "free_count", "lens_out", "free_count_out",
                                                     "device_status")]
for _op in ("tables", "release"):
    BAD_ARGS += [(_op, {"B": -1}, "EINVAL"), (_op, {"B": 8193}, "ENOTSUP"), (_op, {"page_size": 12}, "EINVAL"), (_op, {"num_pages": 0}, "EINVAL"),
                 (_op, {"num_pages": 1 << 28}, "EINVAL"), (_op, {"max_pages": 0}, "EINVAL"), (_op, {"max_pages": 1 << 28}, "EINVAL")]
BAD_ARGS += [("tables", {"T": -1}, "EINVAL")]
BAD_ARGS += [(_op, {"T": (1 << 30) + 1}, "EINVAL") for _op in ("tables", "write", "attention")]
BAD_ARGS += [("gather", {"B": 8192, "S_cap": 1 << 23}, "ENOTSUP")]
BAD_ARGS += [("write", {k: 0}, "EINVAL") for k in ("cache", "k", "v", "slots", "device_status", "token_stride", "head_stride")]
BAD_ARGS += [("write", {"k": P + 8}, "EINVAL"), ("write", {"v": P + 4}, "EINVAL"), ("write", {"T": -1}, "EINVAL"),
             ("write", {"token_stride": 1028}, "EINVAL"), ("write", {"head_stride": -128}, "EINVAL")]
BAD_ARGS += [("gather", {k: 0}, "EINVAL") for k in ("cache", "block_table", "lens", "out_K", "out_V", "device_status", "S_cap", "max_pages")]
BAD_ARGS += [("gather", {"out_K": P + 8}, "EINVAL"), ("gather", {"B": -1}, "EINVAL"), ("gather", {"B": 8193}, "ENOTSUP")]
BAD_ARGS += [("attention", {k: 0}, "EINVAL") for k in ("cache", "q", "cu_new", "kv_lens", "block_table", "out", "workspace", "device_status",
                                                       "max_pages", "q_token_stride", "out_head_stride")]
BAD_ARGS += [("attention", {"q": P + 2}, "EINVAL"), ("attention", {"out": P + 8}, "EINVAL"), ("attention", {"lse": P + 2}, "EINVAL"),
             ("attention", {"workspace": P + 128}, "EINVAL"), ("attention", {"q_head_stride": 130}, "EINVAL"),
             ("attention", {"out_token_stride": -4096}, "EINVAL"), ("attention", {"H_q": 12}, "EINVAL"), ("attention", {"H_q": 0}, "EINVAL"),
             ("attention", {"H_q": 8 * 129}, "ENOTSUP"), ("attention", {"scale": -0.5}, "EINVAL"), ("attention", {"scale": float("nan")}, "EINVAL"),
             ("attention", {"scale": float("inf")}, "EINVAL"), ("attention", {"window": -1}, "EINVAL"), ("attention", {"B": -1}, "EINVAL"),
             ("attention", {"T": -1}, "EINVAL"), ("attention", {"B": 8193}, "ENOTSUP"), ("attention", {"workspace_bytes": 100}, "ENOMEM"),
             ("attention", {"max_pages": 1 << 28}, "EINVAL")]


@pytest.mark.parametrize("op,bad,want", BAD_ARGS, ids=lambda x: str(x))
def test_refused_arguments(kv, op, bad, want):
    cache, ops = calls(kv)
    fn, good = ops[op]
    assert kv.STATUS_NAMES[fn(**{**good, **bad})] == want


@pytest.mark.parametrize("op", ["write", "gather", "attention"])
@pytest.mark.parametrize("bad,want", BAD_CACHES, ids=lambda x: str(x))
def test_refused_caches(kv, op, bad, want):
    _, ops = calls(kv)
    fn, good = ops[op]
    d = desc(kv, **bad)
    assert kv.STATUS_NAMES[fn(**{**good, "cache": C.addressof(d)})] == want


def test_nothing_to_do_is_no_error(kv):
    _, ops = calls(kv)
    for op, none in (("write", {"T": 0}), ("gather", {"B": 0}), ("attention", {"T": 0}), ("attention", {"B": 0})):
        fn, good = ops[op]
        assert fn(**{**good, **none}) == kv.OK


def test_workspace_query(kv):
    assert kv.kvev_paged_attention_workspace(32, 8, 128) >= kv.PAGED_SYNC_BYTES
    for args, want in (((32, 5, 128), kv.EINVAL), ((0, 1, 128), kv.EINVAL), ((8, 0, 128), kv.EINVAL), ((8, 8, 80), kv.ENOTSUP),
                       ((129, 1, 64), kv.ENOTSUP)):
        with pytest.raises(kv.KvevError) as e:
            kv.kvev_paged_attention_workspace(*args)
        assert e.value.code == want
    assert kv.load().kvev_paged_attention_workspace(8, 8, 64, None) == kv.EINVAL
