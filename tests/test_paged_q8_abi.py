"""What the kvev_paged_q8_* and kvev_paged_attention_shared entry points refuse, before any device work (no GPU needed)."""
import ctypes as C

import pytest
import torch

from tests import q8_ref
from tests.test_paged_abi import desc as desc16

P = 1 << 20  # stands for a device pointer: 16-byte aligned, never read by the host


@pytest.fixture(scope="module")
def kv():
    from paper_2606_15157_gb300 import build, kvev
    build.build()
    kvev.load()
    return kvev


def desc(kv, **kw):
    a = {"K": P, "V": P, "K_scale": P, "V_scale": P, "page_stride": 16 * 8 * 128, "token_stride": 8 * 128, "head_stride": 128,
         "scale_page_stride": 128, "num_pages": 64, "page_size": 16, "H_kv": 8, "d": 128, "dtype": kv.BF16, **kw}
    return kv.PagedQ8CacheDesc(*[a[n] for n, _ in kv.PagedQ8CacheDesc._fields_])


BAD_CACHES = [({"K": 0}, "EINVAL"), ({"V": 0}, "EINVAL"), ({"K_scale": 0}, "EINVAL"), ({"V_scale": 0}, "EINVAL"), ({"K": P + 8}, "EINVAL"),
              ({"V": P + 2}, "EINVAL"), ({"page_stride": 0}, "EINVAL"), ({"token_stride": -1024}, "EINVAL"), ({"head_stride": 136}, "EINVAL"),
              ({"scale_page_stride": 127}, "EINVAL"), ({"scale_page_stride": -128}, "EINVAL"), ({"num_pages": 0}, "EINVAL"),
              ({"page_size": 24}, "EINVAL"), ({"page_size": 4}, "EINVAL"), ({"page_size": 512}, "EINVAL"), ({"num_pages": 1 << 27}, "EINVAL"),
              ({"H_kv": 0}, "EINVAL"), ({"d": 96}, "ENOTSUP"), ({"dtype": 2}, "EINVAL")]


def calls(kv):
    cache, plain = desc(kv), desc16(kv)
    at, at16 = C.addressof(cache), C.addressof(plain)
    need = kv.kvev_paged_attention_workspace(32, 8, 128)
    attn = dict(cache=at, q=P, q_token_stride=4096, q_head_stride=128, cu_new=P, kv_lens=P, block_table=P, max_pages=8, B=4, T=9, H_q=32,
                scale=0.0, window=0, out=P, out_token_stride=4096, out_head_stride=128, lse=P, workspace=P, workspace_bytes=need,
                device_status=P, stream=None)
    shared = {**attn, "cache": at16, "groups": P, "shared_lens": P, "N": 2,
              "workspace_bytes": kv.kvev_paged_attention_shared_workspace(32, 8, 128, 9)}
    del shared["window"]
    return (cache, plain), {
        "write": (kv.kvev_paged_q8_write, dict(cache=at, k=P, v=P, token_stride=1024, head_stride=128, slots=P, T=9, device_status=P, stream=None)),
        "gather": (kv.kvev_paged_q8_gather, dict(cache=at, block_table=P, max_pages=8, lens=P, B=4, S_cap=128, out_K=P, out_V=P,
                                                 device_status=P, stream=None)),
        "attention": (kv.kvev_paged_q8_attention, attn), "shared": (kv.kvev_paged_attention_shared, shared)}


BAD_ARGS = [("write", {k: 0}, "EINVAL") for k in ("cache", "k", "v", "slots", "device_status", "token_stride", "head_stride")]
BAD_ARGS += [("write", {"k": P + 8}, "EINVAL"), ("write", {"v": P + 4}, "EINVAL"), ("write", {"T": -1}, "EINVAL"),
             ("write", {"T": (1 << 30) + 1}, "EINVAL"), ("write", {"token_stride": 1028}, "EINVAL"), ("write", {"head_stride": -128}, "EINVAL")]
BAD_ARGS += [("gather", {k: 0}, "EINVAL") for k in ("cache", "block_table", "lens", "out_K", "out_V", "device_status", "S_cap", "max_pages")]
BAD_ARGS += [("gather", {"out_K": P + 8}, "EINVAL"), ("gather", {"B": -1}, "EINVAL"), ("gather", {"B": 8193}, "ENOTSUP"),
             ("gather", {"max_pages": 1 << 28}, "EINVAL"), ("gather", {"B": 8192, "S_cap": 1 << 23}, "ENOTSUP")]
for _op in ("attention", "shared"):
    BAD_ARGS += [(_op, {k: 0}, "EINVAL") for k in ("cache", "q", "cu_new", "kv_lens", "block_table", "out", "workspace", "device_status",
                                                   "max_pages", "q_token_stride", "out_head_stride")]
    BAD_ARGS += [(_op, {"q": P + 2}, "EINVAL"), (_op, {"out": P + 8}, "EINVAL"), (_op, {"lse": P + 2}, "EINVAL"),
                 (_op, {"workspace": P + 128}, "EINVAL"), (_op, {"q_head_stride": 130}, "EINVAL"), (_op, {"out_token_stride": -4096}, "EINVAL"),
                 (_op, {"H_q": 12}, "EINVAL"), (_op, {"H_q": 0}, "EINVAL"), (_op, {"H_q": 8 * 129}, "ENOTSUP"), (_op, {"scale": -0.5}, "EINVAL"),
                 (_op, {"scale": float("nan")}, "EINVAL"), (_op, {"scale": float("inf")}, "EINVAL"), (_op, {"B": -1}, "EINVAL"),
                 (_op, {"T": -1}, "EINVAL"), (_op, {"T": (1 << 30) + 1}, "EINVAL"), (_op, {"B": 8193}, "ENOTSUP"),
                 (_op, {"workspace_bytes": 100}, "ENOMEM"), (_op, {"max_pages": 1 << 28}, "EINVAL")]
BAD_ARGS += [("attention", {"window": -1}, "EINVAL"), ("shared", {"N": -1}, "EINVAL"), ("shared", {"groups": 0}, "EINVAL"),
             ("shared", {"shared_lens": 0}, "EINVAL"), ("shared", {"N": 8189}, "ENOTSUP"), ("shared", {"T": 100000}, "ENOMEM")]


@pytest.mark.parametrize("op,bad,want", BAD_ARGS, ids=lambda x: str(x))
def test_refused_arguments(kv, op, bad, want):
    held, ops = calls(kv)
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
    held, ops = calls(kv)
    for op, none in (("write", {"T": 0}), ("gather", {"B": 0}), ("attention", {"T": 0}), ("attention", {"B": 0}), ("shared", {"T": 0}),
                     ("shared", {"B": 0}), ("shared", {"B": 0, "N": 0, "groups": 0, "shared_lens": 0})):
        fn, good = ops[op]
        assert fn(**{**good, **none}) == kv.OK


def test_workspace_query(kv):
    at = kv.kvev_paged_attention_shared_workspace
    assert at(32, 8, 128, 0) >= kv.kvev_paged_attention_workspace(32, 8, 128)
    assert at(32, 8, 128, 1000) >= at(32, 8, 128, 0) + 1000 * 32 * 2 * (128 + 1) * 4
    assert at(128, 1, 128, 1 << 30) > 1 << 47  # counted in 64 bits
    for args, want in (((32, 5, 128, 1), kv.EINVAL), ((0, 1, 128, 1), kv.EINVAL), ((8, 8, 128, -1), kv.EINVAL), ((8, 8, 80, 1), kv.ENOTSUP),
                       ((129, 1, 64, 1), kv.ENOTSUP)):
        with pytest.raises(kv.KvevError) as e:
            at(*args)
        assert e.value.code == want
    assert kv.load().kvev_paged_attention_shared_workspace(8, 8, 64, 1, None) == kv.EINVAL


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rows_read_back_are_the_nearest_their_codes_allow(dtype):
    """The plain form that the GPU tests go by, by what must hold of it: an element is off by at most half a step of e4m3 (2^-4
    of it, or 2^-10 of the row's power of two), its value is one of the 16-bit type, and a second time gives the same codes."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn((400, 64), generator=g) * torch.exp2(torch.randint(-14, 14, (400, 1), generator=g).float())
    x = x.to(dtype)
    x[0], x[1, :] = 0, torch.finfo(dtype).max
    x[2] = torch.finfo(dtype).smallest_normal
    codes, b = q8_ref.quantise(x)
    v = codes.view(q8_ref.E4M3).double() * torch.exp2(b.double() - 127)[:, None]
    assert torch.equal(v.to(dtype).double(), v)
    err, step = (v - x.double()).abs(), torch.exp2(b.double() - 127)[:, None]
    assert (err <= torch.maximum(x.double().abs() * 2.0 ** -4, step * 2.0 ** -10)).all()
    again = q8_ref.quantise(v.to(dtype))
    assert torch.equal(again[0].view(q8_ref.E4M3).double() * torch.exp2(again[1].double() - 127)[:, None], v)
    x[5, 3], x[6, 1] = float("nan"), float("inf")
    codes2, b2 = q8_ref.quantise(x)
    assert codes2[5, 3] == codes2[6, 1] == 0x7f and torch.equal(codes2[7:], codes[7:])
