"""The paged cache's entry points refuse bad arguments on the host, before a GPU
is touched; the float64 definitions that the GPU tests use hold on worked cases."""
import ctypes
import os

import pytest

torch = pytest.importorskip("torch")

import paged_ref as ref  # noqa: E402
from paper_2506_15745_gb300 import build as ipv_build  # noqa: E402
from paper_2506_15745_gb300 import ipv  # noqa: E402
from paper_2506_15745_gb300.paged import PagedBatch, PagedCache  # noqa: E402


@pytest.fixture(scope="module")
def lib():
    ipv_build.build()
    return ipv.load()


PAGES = dict(format=ipv.IPV_PAGES_BF16, n_kv_heads=4, head_dim=128, page_size=64, n_pages=10, page_stride=256,
             head_stride=64, row_stride=1, k=0x10000, v=0x20000, k_par=0x30000, v_par=0x40000)
BATCH = dict(n_seqs=2, max_pages=4, table=0x1000, table_stride=4, row_start=0x2000, kv_len=0x3000, total_rows=5,
             max_rows=3, max_kv=256)
ARGS = dict(q=0x50000, out=0x60000, lse=None, q_row_stride=3584, q_head_stride=128, out_row_stride=3584,
            out_head_stride=128, n_q_heads=28, scale=0.1, causal=1, window=0, sinks=0, workspace=None, workspace_bytes=0)

BAD_PAGES = [dict(format=3), dict(format=-1), dict(n_kv_heads=0), dict(n_kv_heads=70000), dict(head_dim=0), dict(head_dim=136),
             dict(head_dim=100), dict(format=1, head_dim=80), dict(format=2, head_dim=32), dict(page_size=0),
             dict(page_size=48), dict(page_size=8), dict(n_pages=0), dict(n_pages=1 << 31), dict(page_stride=-1),
             dict(head_stride=-64), dict(page_stride=0), dict(head_stride=0), dict(row_stride=0), dict(row_stride=1 << 32), dict(page_stride=1 << 60), dict(k=None), dict(v=None),
             dict(k=0x10008), dict(v=0x10000), dict(format=1, k_par=None), dict(format=2, v_par=0x40004),
             dict(format=1, v_par=0x30000)]
BAD_BATCH = [dict(n_seqs=-1), dict(n_seqs=65536), dict(max_pages=0), dict(table=None), dict(table=0x1002),
             dict(table_stride=3), dict(row_start=None), dict(kv_len=None), dict(kv_len=0x3002), dict(total_rows=-1),
             dict(total_rows=1 << 31), dict(max_rows=-1), dict(max_kv=-1)]
BAD_ARGS = [dict(q=None), dict(out=None), dict(out=0x50000), dict(q=0x50008), dict(q_row_stride=3580),
            dict(out_head_stride=-128), dict(n_q_heads=27), dict(n_q_heads=0), dict(scale=float("nan")),
            dict(scale=float("inf")), dict(causal=2), dict(window=-1), dict(sinks=-1), dict(window=5, causal=0),
            dict(lse=0x70002)]


def refs(pages, batch):
    return ctypes.byref(ipv.PagesDesc(**pages)), ctypes.byref(ipv.Batch(**batch))


@pytest.mark.parametrize("bad", BAD_PAGES + BAD_BATCH, ids=str)
def test_bad_pages_and_batches(lib, bad):
    pages = {**PAGES, **{k: v for k, v in bad.items() if k in PAGES}}
    batch = {**BATCH, **{k: v for k, v in bad.items() if k in BATCH}}
    p, b = refs(pages, batch)
    args, n = ipv.AttendArgs(**ARGS), ctypes.c_int64(5)
    assert lib.ipv_pages_write(p, b, 0x80000, 0x90000, 512, 128, None) == ipv.IPV_EINVAL
    assert lib.ipv_pages_read(p, b, 0x80000, 0x90000, 512, 128, None) == ipv.IPV_EINVAL
    assert lib.ipv_attend(p, b, ctypes.byref(args), None) == ipv.IPV_EINVAL
    assert lib.ipv_attend_workspace(p, b, ctypes.byref(args), ctypes.byref(n)) == ipv.IPV_EINVAL
    assert lib.ipv_last_error().startswith(b"IPV_EINVAL")


@pytest.mark.parametrize("bad", BAD_ARGS, ids=str)
def test_bad_attend_arguments(lib, bad):
    p, b = refs(PAGES, BATCH)
    assert lib.ipv_attend(p, b, ctypes.byref(ipv.AttendArgs(**{**ARGS, **bad})), None) == ipv.IPV_EINVAL


@pytest.mark.parametrize("scale", [2.4e38, -2.4e38, 3.4e38])
def test_a_scale_that_overflows_in_the_kernels_base_is_refused(lib, scale):
    """The kernels work with scale * log2(e)."""
    p, b = refs(PAGES, BATCH)
    assert lib.ipv_attend(p, b, ctypes.byref(ipv.AttendArgs(**{**ARGS, "scale": scale})), None) == ipv.IPV_EINVAL


@pytest.mark.parametrize("fmt", [ipv.IPV_PAGES_U8, ipv.IPV_PAGES_U4])
def test_a_workspace_that_no_number_holds_is_refused(lib, fmt):
    """Codes and many query rows: n_seqs * heads * max_kv rows of 2 * dim bytes, K and V. 2^70 bytes come out as 0 or as
    anything in 64 bits, and the kernels would write behind a workspace of that size."""
    p, b = refs({**PAGES, "format": fmt, "n_kv_heads": 65535, "page_size": 1 << 30, "n_pages": 65535, "page_stride": 1, "head_stride": 1},
                {**BATCH, "n_seqs": 65535, "max_pages": 1, "table": None, "table_stride": 1, "max_kv": 1 << 30, "max_rows": 65, "total_rows": 65})
    args = ipv.AttendArgs(**{**ARGS, "n_q_heads": 65535})
    n = ctypes.c_int64(0)
    assert lib.ipv_attend_workspace(p, b, ctypes.byref(args), ctypes.byref(n)) == ipv.IPV_EINVAL
    assert lib.ipv_attend(p, b, ctypes.byref(args), None) == ipv.IPV_EINVAL


def test_null_structures_and_bad_rows(lib):
    p, b = refs(PAGES, BATCH)
    args, n = ctypes.byref(ipv.AttendArgs(**ARGS)), ctypes.c_int64(0)
    assert lib.ipv_attend(None, b, args, None) == ipv.IPV_EINVAL
    assert lib.ipv_attend(p, None, args, None) == ipv.IPV_EINVAL
    assert lib.ipv_attend(p, b, None, None) == ipv.IPV_EINVAL
    assert lib.ipv_attend_workspace(p, b, args, None) == ipv.IPV_EINVAL
    for rows in ((None, 0x90000, 512, 128), (0x80000, None, 512, 128), (0x80008, 0x90000, 512, 128),
                 (0x80000, 0x90000, 516, 128), (0x80000, 0x90000, 512, -8)):
        assert lib.ipv_pages_write(p, b, *rows, None) == ipv.IPV_EINVAL
        assert lib.ipv_pages_read(p, b, *rows, None) == ipv.IPV_EINVAL
    assert lib.ipv_pages_read(p, b, 0x80000, 0x80000, 512, 128, None) == ipv.IPV_EINVAL


def test_diagnostics(lib):
    assert lib.ipv_attend_error(None) == ipv.IPV_EINVAL
    assert lib.ipv_attend_wait_limit(-1) == ipv.IPV_EINVAL
    assert lib.ipv_attend_wait_limit(0) == ipv.IPV_OK


def test_an_empty_batch_is_nothing_to_do(lib):
    for empty in (dict(n_seqs=0, row_start=None, kv_len=None), dict(max_rows=0), dict(total_rows=0)):
        p, b = refs(PAGES, {**BATCH, **empty})
        args, n = ipv.AttendArgs(**ARGS), ctypes.c_int64(5)
        assert lib.ipv_pages_write(p, b, 0x80000, 0x90000, 512, 128, None) == ipv.IPV_OK
        assert lib.ipv_pages_read(p, b, 0x80000, 0x90000, 512, 128, None) == ipv.IPV_OK
        assert lib.ipv_attend(p, b, ctypes.byref(args), None) == ipv.IPV_OK
        assert lib.ipv_attend_workspace(p, b, ctypes.byref(args), ctypes.byref(n)) == ipv.IPV_OK and n.value == 0


def test_a_page_of_any_size_for_one_page_per_sequence(lib):
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    p, b = refs({**PAGES, "page_size": 9408}, {**BATCH, "max_pages": 1, "table": None, "table_stride": 1})
    n = ctypes.c_int64(0)  # accepted: what fails is the missing GPU
    assert lib.ipv_attend_workspace(p, b, ctypes.byref(ipv.AttendArgs(**ARGS)), ctypes.byref(n)) == ipv.IPV_ECUDA


def test_the_binding_checks_tensors():
    cpu = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        PagedCache.from_tensors("bf16", cpu, cpu)
    with pytest.raises(ValueError):
        PagedCache.from_tensors("f8", cpu, cpu)
    with pytest.raises(ValueError):
        PagedBatch(None, torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), total_rows=1, max_rows=1, max_kv=1)


# ------------------------------------------------ the definitions, on worked cases
def test_quantise_worked_case():
    # 64 values 0..63 in 4 bits: m = 0, s = 63/15 = 4.2 rounded up to fp16 (spacing 2^-8): 4.203125
    x = torch.arange(64, dtype=torch.float32).bfloat16()[None]
    u, s, m = ref.quantise(x, "u4")
    assert float(s) == 4.203125 and float(m) == 0.0
    assert u[0, 0] == 0 and u[0, 63] == 15 and u[0, 21] == 5 and u[0, 2] == 0 and u[0, 3] == 1
    assert float(ref.values(u, s, m)[0, 63]) == 15 * 4.203125


def test_rounding_to_fp16_is_directed():
    x = torch.tensor([1.0, 1.0 + 2.0 ** -12, -1.0 - 2.0 ** -12, 1e-9, -1e-9, 0.0], dtype=torch.float64)
    assert ref.f16_round(x, True).double().tolist() == [1.0, 1.0 + 2.0 ** -10, -1.0, 2.0 ** -24, 0.0, 0.0]
    assert ref.f16_round(x, False).double().tolist() == [1.0, 1.0, -1.0 - 2.0 ** -10, 0.0, -(2.0 ** -24), 0.0]


def test_pack_places_words():
    u = torch.arange(128)
    b = ref.pack(u, "u8")
    # word of channels 4(t + 4w).. in place 4t + w: t = 1, w = 2 holds channels 36..39 at bytes 24..27
    assert b[24:28].tolist() == [36, 37, 38, 39] and b[64 + 24] == 100
    b = ref.pack(torch.arange(64) % 16, "u4")
    # word of channels 8(t + 4w).. in place 2t + w: t = 3, w = 1 holds channels 56..63 at bytes 28..31
    assert b[28:32].tolist() == [(9 << 4) | 8, (11 << 4) | 10, (13 << 4) | 12, (15 << 4) | 14]


def test_attend_worked_case():
    # two equal keys: the mean of their values; with a window of 1, the last one alone
    q = torch.ones(1, 1, 8, dtype=torch.float64)
    k = torch.ones(2, 1, 8, dtype=torch.float64)
    v = torch.stack([torch.zeros(1, 8), torch.ones(1, 8)]).double()
    out, lse, _, _ = ref.attend(q, k, v, 0.5)
    assert torch.allclose(out, torch.full_like(out, 0.5)) and torch.allclose(lse, torch.log(2 * torch.exp(torch.tensor(4.0).double())))
    out, lse, _, _ = ref.attend(q, k, v, 0.5, window=1)
    assert torch.equal(out, torch.ones_like(out)) and float(lse) == 4.0
    assert ref.sees(5, 2, True, 2, 1).tolist() == [[True, False, True, True, False], [True, False, False, True, True]]
    assert not ref.sees(3, 5, True, 0, 0)[:2].any()


def test_overlapping_kernels_read_coherently():
    """The paged cache's kernels are launched before their predecessors end, which may still be writing what they are
    about to read: no loads through the path that is for memory nobody writes while the kernel is there."""
    for name in ("paged_rows.cu", "attend_rows.cu", "attend_tiles.cu", "attend_share.cuh", "paged.cuh"):
        with open(os.path.join(ipv_build.CSRC, name)) as f:
            text = f.read()
        for banned in ("ld_stream(", "ld.global.nc", "__ldg("):
            assert banned not in text, (name, banned)
