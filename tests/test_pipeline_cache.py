"""What RotaryTable and PagedCache hand to the library, looked at on the host: the calls are recorded, no GPU is needed.  A call whose
tensors do not hold what it would read or write is refused before anything reaches the library."""
import pytest

torch = pytest.importorskip("torch")


@pytest.fixture
def host(monkeypatch):
    """pipeline with recorded library calls; its objects live on the CPU."""
    from paper_2609_29812_b200 import binding as B, pipeline as P
    calls = []

    def record(name, result=0):
        def call(*args, **kw):
            calls.append((name, args, kw))
            return result
        return call
    for name in ("fl_rope_table", "fl_rotate_rows", "fl_cache_append", "fl_cache_read", "fl_cache_attention"):
        monkeypatch.setattr(B, name, record(name))
    monkeypatch.setattr(B, "fl_cache_attention_workspace_bytes", lambda *a: 256)
    monkeypatch.setattr(B, "_stream_of", lambda index: P.__dict__.get("test_stream"))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(P, "status_word", lambda dev: torch.zeros(1, dtype=torch.int32))
    return P, B, calls


def refused(B, calls, f):
    n = len(calls)
    with pytest.raises(B.FlashLoopError) as e:
        f()
    assert e.value.status == B.FL_ERR_INVALID_ARG and len(calls) == n


BF16, F32, F16 = torch.bfloat16, torch.float32, torch.float16


def rows(n, heads=2, dim=64, dtype=BF16):
    return torch.zeros(n, heads, dim, dtype=dtype)


def test_rotation_takes_what_it_reads(host):
    P, B, calls = host
    t = P.RotaryTable(None, 100, 64, device="cpu")
    pos = torch.arange(5, dtype=torch.int32)
    for x in (rows(5, dtype=F16), rows(5, dtype=torch.float64), rows(5).view(5, 128), rows(5).transpose(1, 2), rows(1).expand(5, 2, 64), rows(5, 4)[:, ::2],
              torch.zeros(600, dtype=BF16).as_strided((5, 2, 64), (100, 64, 1)), rows(5).to("meta")):
        refused(B, calls, lambda: t.rotate(x, pos))
    for p in (pos.long(), pos[:4], pos.view(5, 1), torch.arange(10, dtype=torch.int32)[::2], pos.float(), pos.to("meta")):
        refused(B, calls, lambda: t.rotate(rows(5), p))
    for out in (rows(5, dtype=F32), rows(4), rows(5, 1), rows(5, 2, 32), rows(1).expand(5, 2, 64), rows(5).to("meta")):
        refused(B, calls, lambda: t.rotate(rows(5), pos, out=out))
    # what it takes: both types, parts of longer rows, a single row of any stride, one head of any stride, none at all
    wide = torch.zeros(5, 3, 2, 64, dtype=F32)
    for x, stride in ((rows(5), 128), (wide[:, 1], 384), (rows(5)[:1], 128), (wide[:1, 0], 128), (rows(5, 1).expand(5, 1, 64), 64), (wide[:, 2, :1], 384), (rows(0), 128)):
        out = t.rotate(x, pos)
        name, args, _ = calls[-1]
        assert name == "fl_rotate_rows" and args[1] is x and args[2] == stride and args[7] == (B.FL_F32 if x.dtype == F32 else B.FL_BF16)
        assert out.shape == x.shape and out.dtype == x.dtype and args[10] is out


def test_a_cache_has_a_storage_type_and_a_code(host):
    P, B, calls = host
    for bad in (dict(dtype=F16), dict(dtype=torch.int8), dict(code=2)):
        refused(B, calls, lambda: P.PagedCache(None, 1, 1, 64, 100, device="cpu", **bad))


@pytest.mark.parametrize("dtype,other", [(BF16, F32), (F32, BF16)])
def test_append_takes_what_it_reads(host, dtype, other):
    P, B, calls = host
    c = P.PagedCache(None, 3, 2, 64, 100, page=16, dtype=dtype, device="cpu")
    r = lambda n, heads=2, dim=64: rows(n, heads, dim, dtype)
    new = [3, 0, 4]
    for bad in (rows(7, dtype=other), rows(7, dtype=F16), r(6), r(7, 1), r(7, 4), r(7, 2, 128), r(1).expand(7, 2, 64), r(7, 2, 128)[:, :, ::2], r(7).view(7, 128), r(7).to("meta")):
        refused(B, calls, lambda: c.append(bad, r(7), new))
        refused(B, calls, lambda: c.append(r(7), bad, new))
    for bad in ([3, 4], [3, 0, 4, 0], [8, 0, -1], []):
        refused(B, calls, lambda: c.append(r(7), r(7), bad))
    for bad in (torch.arange(7), torch.arange(6, dtype=torch.int32), torch.arange(14, dtype=torch.int32)[::2]):
        refused(B, calls, lambda: c.append(r(7), r(7), new, pos=bad))
    t = P.RotaryTable(None, 100, 64, device="cpu")
    t.table = t.table.to("meta")
    n = len(calls)
    refused(B, calls, lambda: c.append(r(7), r(7), new, t))
    assert c.lens == [0, 0, 0] and len(calls) == n
    slab = torch.zeros(7, 3, 2, 64, dtype=dtype)
    starts = c.append(slab[:, 1], slab[:, 2], new)
    name, args, _ = calls[-1]
    assert name == "fl_cache_append" and args[4] == args[6] == 384 and args[8] == 7 and starts.tolist() == [0, 3, 3, 7] and c.lens == new


def test_attend_and_read_take_what_they_read(host):
    P, B, calls = host
    c = P.PagedCache(None, 2, 2, 64, 100, page=16, device="cpu")
    new = [2, 3]
    starts = torch.tensor([0, 2, 5], dtype=torch.int32)
    for bad in (rows(5, 4, dtype=F32), rows(5, 4, 128), rows(4, 4), rows(6, 4), rows(1, 4).expand(5, 4, 64), rows(5, 8)[:, ::2], rows(5, 4).to("meta")):
        refused(B, calls, lambda: c.attend(bad, new, 0.125))
    for bad in (rows(4, 4), rows(5, 4, 128)):
        refused(B, calls, lambda: c.attend(bad, new, 0.125, starts))
    for bad in ([5], [2, 3, 0], [6, -1]):
        refused(B, calls, lambda: c.attend(rows(5, 4), bad, 0.125))
    for bad in (starts.long(), starts[:2], starts.view(1, 3), starts.to("meta")):
        refused(B, calls, lambda: c.attend(rows(5, 4), new, 0.125, bad))
    for b, first, n in ((2, 0, 1), (-1, 0, 1), (0, -1, 1), (0, 0, -1), (0, 1, None)):
        refused(B, calls, lambda: c.read(b, first, n))
    o, lse = c.attend(rows(5, 4), new, 0.125)
    assert calls[-1][0] == "fl_cache_attention" and o.shape == (5, 4, 64) and lse.shape == (5, 4)
    o, _ = c.attend(rows(9, 4), new, 0.125, starts + 4)                   # rows of a longer tensor
    assert calls[-1][1][6] == 9 and o.shape[0] == 9
    k, v = c.read(1, 0, 4)
    assert calls[-1][0] == "fl_cache_read" and k.shape == v.shape == (4, 2, 64)


def test_calls_on_different_streams_share_no_workspace(host, monkeypatch):
    P, B, calls = host
    need, used = [256], []
    monkeypatch.setattr(B, "fl_cache_attention_workspace_bytes", lambda *a: need[0])
    c = P.PagedCache(None, 1, 1, 64, 100, page=16, device="cpu")
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: used.append((self.data_ptr(), s)))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda dev=None: P.test_stream)

    def workspace(stream):
        monkeypatch.setattr(P, "test_stream", stream, raising=False)
        c.attend(rows(1, 1), [1], 0.125)
        assert calls[-1][0] == "fl_cache_attention" and int(calls[-1][1][13]) == calls[-1][1][12].numel()
        return calls[-1][1][12]

    first, second = workspace(None), workspace(7)
    assert first.data_ptr() != second.data_ptr() and workspace(None) is first and workspace(7) is second
    need[0] = 512
    grown = workspace(7)
    assert grown.numel() == 512 and workspace(None).numel() == 512 and workspace(None).data_ptr() != grown.data_ptr()
    # lengths that another stream has read are told to the allocator before the object lets go of them
    assert used and all(u == (c.len_dev.data_ptr(), 7) for u in used)
    # a captured call's workspace is the graph's
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    own = workspace(7)
    assert own is not grown and workspace(7) is not own
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    assert workspace(7) is grown


def test_a_reservation_that_cannot_be_met_takes_no_page(host):
    P, B, calls = host
    c = P.PagedCache(None, 3, 1, 64, 64, n_pages=5, page=16, device="cpu")
    for new in ([32, 0, 65], [33, 32, 32], [0, 80, 0]):                       # more pages than are free, or than a sequence's table holds
        with pytest.raises(RuntimeError):
            c.append(rows(sum(new), 1), rows(sum(new), 1), new)
        assert len(c.free) == 5 and c.pages == [[], [], []] and c.lens == [0, 0, 0]
    c.append(rows(80, 1), rows(80, 1), [33, 31, 16])
    assert [len(p) for p in c.pages] == [2, 1, 1] and len(c.free) == 1
    c.append(rows(1, 1), rows(1, 1), [0, 1, 0])
    assert not c.free and c.page_table[1, :2].tolist() == c.pages[1]


def test_a_rotation_hears_of_positions_outside_its_table(host):
    P, B, calls = host
    t = P.RotaryTable(None, 100, 64, device="cpu")
    t.rotate(rows(1), torch.tensor([100], dtype=torch.int32))
    assert calls[-1][0] == "fl_rotate_rows" and calls[-1][2]["status"] is t.status
    t.check_status()
    t.status.fill_(B.FL_ERR_INVALID_ARG)                                       # as the kernel does
    with pytest.raises(B.FlashLoopError) as e:
        t.check_status()
    assert e.value.status == B.FL_ERR_INVALID_ARG
