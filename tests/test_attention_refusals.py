"""What attention and the cache's pages refuse: every check comes before the GPU is touched, so the pointers here are never read."""
import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2412_00099_amd import binding

    return binding


P = 0x10000  # never dereferenced


def refused(B, call, good, **bad):
    args = dict(good, **bad)
    code = call(*args.values())
    assert code == B.MOE_EINVAL, (bad, code)
    assert B.moe_last_error()


PLAN = dict(have=P, more=P, n_seqs=3, page=16, free=P, n_free=8, used=None, table=P, table_pages=4, offsets=P, slots=P, positions=P, n_tokens=9,
            lengths=2 * P, used_out=P, stream=None)


@pytest.mark.parametrize("bad", [
    dict(have=None), dict(more=None), dict(free=None), dict(table=None), dict(offsets=None), dict(slots=None), dict(positions=None), dict(lengths=None),
    dict(used_out=None), dict(n_seqs=-1), dict(n_seqs=16385), dict(page=0), dict(page=8), dict(page=17), dict(page=2048), dict(page=-16), dict(n_free=-1),
    dict(table_pages=-1), dict(n_tokens=-1), dict(n_tokens=1 << 26), dict(have=P + 2), dict(used=P + 1), dict(used=P), dict(lengths=P), dict(table=P + 1)])
def test_plan(B, bad):
    refused(B, B.lib.moe_plan_pages, PLAN, **bad)


CACHE = dict(k_pages=P, v_pages=P, cache_fmt=1, page_stride=2 * 16 * 64, n_pages=9, page=16, k_scale=None, v_scale=None)
BAD_CACHE = [dict(k_pages=None), dict(v_pages=None), dict(cache_fmt=0), dict(cache_fmt=3), dict(page_stride=2 * 16 * 64 - 8), dict(page_stride=2 * 16 * 64 + 4),
             dict(page_stride=(1 << 40) + 16), dict(n_pages=-1), dict(n_pages=1 << 27), dict(page=24), dict(page=8), dict(page=2048), dict(k_scale=P),
             dict(v_scale=P), dict(cache_fmt=2), dict(cache_fmt=2, k_scale=P), dict(cache_fmt=2, k_scale=P + 2, v_scale=P), dict(k_pages=P + 8),
             dict(cache_fmt=2, k_scale=P, v_scale=P, page_stride=2 * 16 * 64 + 8)]
STORE = dict(k=P, v=P, fmt=1, k_stride=128, k_head=64, v_stride=128, v_head=64, slots=P, n_rows=5, kv=2, dim=64,
             **{k: CACHE[k] for k in ("k_pages", "v_pages", "cache_fmt", "page_stride", "n_pages", "page", "k_scale", "v_scale")}, stream=None)


@pytest.mark.parametrize("bad", BAD_CACHE + [dict(k=None), dict(v=None), dict(slots=None), dict(fmt=2), dict(fmt=-1), dict(n_rows=-1), dict(n_rows=1 << 26), dict(kv=0),
                                             dict(kv=257), dict(dim=0), dict(dim=60), dict(dim=136), dict(k=P + 1), dict(slots=P + 2), dict(k_stride=-1), dict(v_head=-8)])
def test_store(B, bad):
    refused(B, B.lib.moe_store_pages, STORE, **bad)


SEEN = dict(softmax_scale=0.125, window=0, sinks=0)
BAD_SEEN = [dict(softmax_scale=0.0), dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")), dict(window=-1), dict(sinks=-1)]
PAGES = dict(q=P, q_stride=256, q_head=64, **CACHE, table=P, table_pages=4, lengths=P, n_seqs=3, heads=4, kv=2, dim=64, **SEEN, y=P, work=P,
             work_bytes=1 << 28, stream=None)


@pytest.mark.parametrize("bad", BAD_CACHE + BAD_SEEN + [
    dict(q=None), dict(table=None), dict(lengths=None), dict(y=None), dict(work=None), dict(work_bytes=100), dict(work=P + 8), dict(heads=5), dict(heads=0),
    dict(heads=512), dict(kv=0), dict(kv=-2), dict(dim=4), dict(dim=256), dict(n_seqs=-1), dict(n_seqs=16385), dict(table_pages=-1), dict(q_stride=63),
    dict(q_stride=260), dict(q_stride=1 << 24), dict(q_head=32), dict(q_head=68), dict(q=P + 8), dict(y=P + 2), dict(lengths=P + 1)])
def test_pages(B, bad):
    refused(B, B.lib.moe_attend_pages, PAGES, **bad)


ROWS = dict(q=P, q_stride=256, q_head=64, k=P, k_stride=128, k_head=64, v=P, v_stride=128, v_head=64, offsets=P, k_offsets=P, n_seqs=3, n_rows=100,
            n_k_rows=300, heads=4, kv=2, dim=64, **SEEN)
BAD_ROWS = BAD_SEEN + [
    dict(q=None), dict(k=None), dict(v=None), dict(offsets=None), dict(k_offsets=None), dict(n_seqs=-1), dict(n_seqs=16385), dict(n_rows=-1),
    dict(n_rows=1 << 26), dict(n_k_rows=1 << 26), dict(heads=3), dict(dim=12), dict(dim=136), dict(q_stride=8), dict(k_stride=132), dict(v_head=4),
    dict(v_stride=1 << 24), dict(q=P + 2), dict(v=P + 8), dict(offsets=P + 2)]


@pytest.mark.parametrize("bad", BAD_ROWS + [dict(y=None), dict(y=P + 4), dict(low=P + 8), dict(lse=P + 2)])
def test_rows(B, bad):
    refused(B, B.lib.moe_attend_rows, dict(ROWS, y=P, low=None, lse=None, work=P, work_bytes=1 << 28, stream=None), **bad)


@pytest.mark.parametrize("bad", [dict(work=None), dict(work=P + 8), dict(work_bytes=1 << 10)])
def test_rows_of_many_keys(B, bad):
    good = dict(ROWS, n_k_rows=9000, y=P, low=None, lse=None, work=P, work_bytes=B.moe_attend_rows_bytes(100, 9000, 3, 4, 2, 64), stream=None)
    refused(B, B.lib.moe_attend_rows, good, **bad)


@pytest.mark.parametrize("bad", BAD_ROWS + [dict(y=None), dict(lse=None), dict(dy=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(dy=P + 8), dict(low=P + 2),
                                            dict(work=None), dict(work=P + 4), dict(work_bytes=100 * 4 * 4)])
def test_rows_backward(B, bad):
    refused(B, B.lib.moe_attend_rows_backward, dict(ROWS, y=P, low=None, lse=P, dy=P, dq=P, dk=P, dv=P, work=P, work_bytes=1 << 30, stream=None), **bad)


def test_workspaces(B):
    size = B.moe_attend_rows_backward_bytes
    assert size(100, 300, 3, 4, 2, 64) >= 1600 and size(0, 0, 0, 4, 2, 64) > 0
    assert all(size(*bad) == 0 for bad in [(-1, 3, 1, 4, 2, 64), (3, 1 << 26, 1, 4, 2, 64), (3, 3, -1, 4, 2, 64), (3, 3, 1, 4, 0, 64), (3, 3, 1, 2, 4, 64), (3, 3, 1, 4, 2, 200)])
    assert size(20001, 20001, 9, 16, 2, 80) < 128 << 20  # (pieces' sums do not grow with the rows)
    size = B.moe_attend_rows_bytes
    assert size(100, 8100, 1, 32, 8, 128) > 0 and size(8192, 8192, 1, 32, 8, 128) == 0 and size(100, 100, 1, 32, 8, 128) == 0
    assert all(size(*bad) == 0 for bad in [(-1, 8100, 1, 4, 2, 64), (3, 1 << 26, 1, 4, 2, 64), (3, 8100, -1, 4, 2, 64), (3, 8100, 0, 4, 2, 64), (0, 8100, 1, 4, 2, 64), (3, 8100, 1, 4, 0, 64)])
    assert max(size(n, 1 << 25, 1, h, 1, 128) for n in (1, 100, 128, 1000, 5000, 32000) for h in (1, 3, 32, 200)) < 80 << 20  # (shares do not grow with the keys)
    assert B.moe_attend_pages_bytes(0, 4, 2, 64) == 0 and B.moe_attend_pages_bytes(3, 4, 2, 64) > 0
    assert B.moe_attend_pages_bytes(3, 4, 0, 64) == 0 and B.moe_attend_pages_bytes(3, 2, 4, 64) == 0


def test_nothing_to_do(B):
    assert B.lib.moe_store_pages(*dict(STORE, n_rows=0, k=None, v=None, slots=None).values()) == B.MOE_OK
    assert B.lib.moe_attend_pages(*dict(PAGES, n_seqs=0, q=None, y=None, work=None, work_bytes=0).values()) == B.MOE_OK
    assert B.lib.moe_attend_rows(*dict(ROWS, n_rows=0, q=None, y=None, low=None, lse=None, work=None, work_bytes=0, stream=None).values()) == B.MOE_OK


def test_tensors_on_the_cpu_and_of_other_shapes(B):
    import paper_2412_00099_amd as moe

    bf16, i32 = torch.bfloat16, torch.int32
    q, k = torch.zeros(5, 4, 64, dtype=bf16), torch.zeros(5, 2, 64, dtype=bf16)
    at = torch.zeros(2, dtype=i32)
    pages, table, n = torch.zeros(3, 2, 16, 64, dtype=bf16), torch.zeros(5, 2, dtype=i32), torch.zeros(5, dtype=i32)
    calls = [
        lambda: moe.attend_rows(q, k, k, at),                                # on the CPU
        lambda: moe.attend_rows(q.float(), k, k, at),
        lambda: moe.attend_rows(q, k, k[:4], at),
        lambda: moe.attend_rows(q, k[..., :32], k[..., :32], at),
        lambda: moe.attend_rows(q[0], k, k, at),
        lambda: moe.attend_rows(q, k, k, at.long()),
        lambda: moe.attend_rows(q, k[:3], k[:3], at),
        lambda: moe.attend_rows(q.transpose(1, 2), k, k, at),
        lambda: moe.attend_rows(q, k, k, at, k_offsets=at[:1]),
        lambda: moe.attend_rows_backward(q, k, k, at, q, moe.KeptAttention(torch.zeros(4, 4), None), q),
        lambda: moe.attend_rows_backward(q, k, k, at, q.float(), moe.KeptAttention(torch.zeros(4, 5), q), q),
        lambda: moe.attend_pages(q, pages, pages, table, n),
        lambda: moe.attend_pages(q, pages, pages[:2], table, n),
        lambda: moe.attend_pages(q, pages, pages.float(), table, n),
        lambda: moe.attend_pages(q, pages.transpose(1, 2), pages.transpose(1, 2), table, n),
        lambda: moe.attend_pages(q, pages, pages, table[:4], n),
        lambda: moe.attend_pages(q, pages, pages, table, n, torch.zeros(3, 2, 8), torch.zeros(3, 2, 16)),
        lambda: moe.store_pages(k, k, n, pages, pages),
        lambda: moe.store_pages(k, k.float(), n, pages, pages),
        lambda: moe.store_pages(q, q, n, pages, pages),
        lambda: moe.store_pages(k, k, n[:4], pages, pages),
        lambda: moe.plan_pages(n, n, table, n, 16, 5),
        lambda: moe.plan_pages(n, n[:4], table, n, 16, 5),
        lambda: moe.plan_pages(n, n, table[:, :1], n, 16, 5),
        lambda: moe.plan_pages(n, n, table, n, 16, 5, used=n),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            print(i)


def test_caches_of_inference_mode_are_not_written_outside_it(B):
    import paper_2412_00099_amd as moe

    k, n = torch.zeros(5, 2, 64, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.int32)
    with torch.inference_mode():
        pages, table = torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(5, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="inference"):
        moe.store_pages(k, k, n, pages, pages)
    with pytest.raises(ValueError, match="inference"):
        moe.plan_pages(n, n, table, n, 16, 5)


def test_each_wrong_shape_or_type_is_told_by_its_own_check(B):
    """These checks come ahead of the one for a GPU, so that each call names what is wrong with it."""
    import paper_2412_00099_amd as moe

    bf16, i32, i8 = torch.bfloat16, torch.int32, torch.int8
    q, k = torch.zeros(5, 4, 64, dtype=bf16), torch.zeros(5, 2, 64, dtype=bf16)
    at, lse = torch.zeros(2, dtype=i32), torch.zeros(4, 5)
    pages, table, n = torch.zeros(3, 2, 16, 64, dtype=bf16), torch.zeros(5, 2, dtype=i32), torch.zeros(5, dtype=i32)
    codes, scale = torch.zeros(3, 2, 16, 64, dtype=i8), torch.zeros(3, 2, 16)
    kept = moe.KeptAttention
    apart = torch.zeros(6, 2, 16, 64, dtype=bf16)[::2]
    calls = [
        (lambda: moe.attend_rows(q, k, k, at), "on a GPU"),
        (lambda: moe.attend_rows(q.float(), k, k, at), "q: Float is not bfloat16"),
        (lambda: moe.attend_rows(q, k.half(), k, at), "k: Half is not bfloat16"),
        (lambda: moe.attend_rows(q, k, k.to(i8), at), "v: Char is not bfloat16"),
        (lambda: moe.attend_rows(q[0], k, k, at), r"q has to be \[tokens, heads, dim\]"),
        (lambda: moe.attend_rows(q, k[:, :, ::2], k, at), r"k has to be \[tokens, heads, dim\] with dense heads"),
        (lambda: moe.attend_rows(q.transpose(1, 2), k, k, at), r"q has to be \[tokens, heads, dim\] with dense heads"),
        (lambda: moe.attend_rows(q, k, k[:4], at), "k and v have to have the same shape"),
        (lambda: moe.attend_rows(q, k[:, :1], k, at), "k and v have to have the same shape"),
        (lambda: moe.attend_rows(q, k[..., :32], k[..., :32], at), "and q their dim"),
        (lambda: moe.attend_rows(q, k[:3], k[:3], at), "without k_offsets"),
        (lambda: moe.attend_rows(q, k, k, at.long()), "offsets has to be contiguous"),
        (lambda: moe.attend_rows(q, k, k, torch.zeros(4, dtype=i32)[::2]), "offsets has to be contiguous"),
        (lambda: moe.attend_rows(q, k, k, torch.zeros(2, 2, dtype=i32)), "offsets has to be"),
        (lambda: moe.attend_rows(q, k, k, at[:0]), "offsets has to be"),
        (lambda: moe.attend_rows(q, k, k, at, k_offsets=at[:1]), "k_offsets has to be contiguous"),
        (lambda: moe.attend_rows(q, k, k, at, k_offsets=at.float()), "k_offsets has to be contiguous"),
        (lambda: moe.attend_rows_backward(q, k, k, at, q, kept(lse, q), q), "on a GPU"),
        (lambda: moe.attend_rows_backward(q, k, k, at, q, kept(lse[:, :4], q), q), "kept.lse has to be contiguous"),
        (lambda: moe.attend_rows_backward(q, k, k, at, q, kept(lse.double(), q), q), "kept.lse has to be contiguous"),
        (lambda: moe.attend_rows_backward(q, k, k, at, q, kept(lse, q[:4]), q), "kept.low has to be contiguous"),
        (lambda: moe.attend_rows_backward(q, k, k, at, q, kept(lse, q.float()), q), "kept.low has to be contiguous"),
        (lambda: moe.attend_rows_backward(q, k, k, at, q.float(), kept(lse, q), q), "y has to be contiguous"),
        (lambda: moe.attend_rows_backward(q, k, k, at, q[:, :2], kept(lse, q), q), "y has to be contiguous"),
        (lambda: moe.attend_rows_backward(q, k, k, at, q, kept(lse, None), q.transpose(0, 1)), "dy has to be contiguous"),
        (lambda: moe.attend_rows_backward(q, k, k, at, q, kept(lse, None), q[:4]), "dy has to be contiguous"),
        (lambda: moe.attend_pages(q, pages, pages, table, n), "on a GPU"),
        (lambda: moe.attend_pages(q, apart, apart, table, n), "on a GPU"),
        (lambda: moe.attend_pages(q.float(), pages, pages, table, n), "q: Float is not bfloat16"),
        (lambda: moe.attend_pages(q, pages, pages[:2], table, n), "k_pages and v_pages have to be"),
        (lambda: moe.attend_pages(q, pages, codes, table, n), "of one type"),
        (lambda: moe.attend_pages(q, pages[0], pages[0], table, n), "k_pages and v_pages have to be"),
        (lambda: moe.attend_pages(q, pages.float(), pages.float(), table, n), "neither bfloat16 nor int8"),
        (lambda: moe.attend_pages(q, pages.transpose(1, 2), pages.transpose(1, 2), table, n), "have to be dense"),
        (lambda: moe.attend_pages(q, pages, apart, table, n), "equally far apart"),
        (lambda: moe.attend_pages(q[..., :32], pages, pages, table, n), "q has another dim"),
        (lambda: moe.attend_pages(q, pages, pages, table[0], n), r"table has to be \[sequences, pages\]"),
        (lambda: moe.attend_pages(q, pages, pages, table[:4], n), "table has to be contiguous"),
        (lambda: moe.attend_pages(q, pages, pages, table[:, :1], n), "table has to be contiguous"),
        (lambda: moe.attend_pages(q, pages, pages, table.long(), n), "table has to be contiguous"),
        (lambda: moe.attend_pages(q, pages, pages, table, n[:4]), "lengths has to be contiguous"),
        (lambda: moe.attend_pages(q, pages, pages, table, n.long()), "lengths has to be contiguous"),
        (lambda: moe.attend_pages(q, codes, codes, table, n, scale[..., :8], scale), "k_scale has to be contiguous"),
        (lambda: moe.attend_pages(q, codes, codes, table, n, scale, scale[:2]), "v_scale has to be contiguous"),
        (lambda: moe.attend_pages(q, codes, codes, table, n, scale, scale.double()), "v_scale has to be contiguous"),
        (lambda: moe.store_pages(k, k, n, pages, pages), "on a GPU"),
        (lambda: moe.store_pages(k.half(), k.half(), n, pages, pages), "k: Half is neither"),
        (lambda: moe.store_pages(k, k.float(), n, pages, pages), "v has to have the shape and type of k"),
        (lambda: moe.store_pages(k, k[:4], n, pages, pages), "v has to have the shape and type of k"),
        (lambda: moe.store_pages(q, q, n, pages, pages), "other heads than k_pages"),
        (lambda: moe.store_pages(k[..., :32], k[..., :32], n, pages, pages), "other heads than k_pages"),
        (lambda: moe.store_pages(k, k, n[:4], pages, pages), "slots has to be contiguous"),
        (lambda: moe.store_pages(k, k, n.long(), pages, pages), "slots has to be contiguous"),
        (lambda: moe.store_pages(k, k, n, codes, codes, scale, scale[..., :8]), "v_scale has to be contiguous"),
        (lambda: moe.plan_pages(n, n, table, n, 16, 5), "on a GPU"),
        (lambda: moe.plan_pages(n, n[:4], table, n, 16, 5), "more has to be contiguous"),
        (lambda: moe.plan_pages(n.long(), n, table, n, 16, 5), "have has to be contiguous"),
        (lambda: moe.plan_pages(n, n, table[:4], n, 16, 5), "table has to be contiguous"),
        (lambda: moe.plan_pages(n, n, table[:, :1], n, 16, 5), "table has to be contiguous"),
        (lambda: moe.plan_pages(n, n, table[0], n, 16, 5), r"table \[sequences, pages\]"),
        (lambda: moe.plan_pages(n, n, table, n.long(), 16, 5), "free has to be contiguous"),
        (lambda: moe.plan_pages(n, n, table, n, 16, 5, used=n), "used has to be contiguous"),
    ]
    for i, (call, what) in enumerate(calls):
        print(i, what)
        with pytest.raises(ValueError, match=what):
            call()
