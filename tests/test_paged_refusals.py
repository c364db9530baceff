"""What the operators around a paged cache refuse: by the C ABI's status codes, before any CUDA call, and by the binding's assertions."""
import ctypes as C
import threading
import time

import pytest
import torch

from paper_2609_09721_b200 import binding

OK, INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = 0, 1, 2, 3, 4
P = 1 << 20         # an address that is never followed


def _rows(heads=8, **more):
    return binding.EfqRows(**{**dict(src=P, dst=P, heads=heads, src_batch=0, src_head=128, src_token=1024, dst_batch=0, dst_head=128, dst_token=1024), **more})


def _cache(**more):
    return binding.EfqPaged(**{**dict(k=P, v=P, k_page=4096, k_head=2048, k_token=128, v_page=4096, v_head=2048, v_token=128, n_pages=10, n_heads=2, page_size=16,
                                      page_table=P, table_stride=4, max_pages=4, cu_seqlens=P, seq_lens=P, n_seqs=3), **more})


def _rotation(**more):
    return binding.EfqRotary(**{**dict(inv_freq=P, n_axes=1, pairs=(C.c_int32 * 4)(64), interleaved=0), **more})


def _attention(rows=None, cache=None, total=10, max_q=1, d=128, dtype=0, scale=0.0, workspace=P, nbytes=1 << 40, lse=None):
    return binding.lib().efq_paged_attention_fwd(rows and C.byref(rows), lse, total, max_q, cache and C.byref(cache), d, dtype, 1, scale, workspace, nbytes, None)


def test_attention_refuses():
    R, K = _rows(), _cache()
    assert _attention(None, K) == INVALID and _attention(R, None) == INVALID
    for bad in (dict(src=None), dict(dst=None), dict(heads=0), dict(heads=7), dict(heads=-2), dict(src_head=-8), dict(dst_token=-8)):
        assert _attention(_rows(**bad), K) == INVALID, bad
    assert _attention(R, K, total=-1) == INVALID and _attention(R, K, max_q=-1) == INVALID
    assert _attention(R, K, scale=float("nan")) == INVALID and _attention(R, K, scale=float("inf")) == INVALID
    for bad in (dict(k=None), dict(v=None), dict(page_table=None), dict(cu_seqlens=None), dict(seq_lens=None), dict(n_pages=0), dict(n_heads=0), dict(max_pages=0),
                dict(n_seqs=-1), dict(table_stride=-1), dict(k_page=-8), dict(v_token=-8)):
        assert _attention(R, _cache(**bad)) == INVALID, bad
    for bad in (8, 24, 0, -16, 8192, 17):
        assert _attention(R, _cache(page_size=bad)) == UNSUPPORTED, bad
    assert _attention(R, _cache(max_pages=1 << 27)) == UNSUPPORTED                   # 2^31 tokens a sequence
    assert _attention(R, K, d=64) == UNSUPPORTED and _attention(R, K, dtype=2) == UNSUPPORTED
    assert _attention(_rows(heads=258), K) == UNSUPPORTED                             # 129 query heads on a KV head
    assert _attention(R, K, total=1 << 31) == UNSUPPORTED
    assert _attention(R, _cache(max_pages=1 << 26, n_seqs=600)) == UNSUPPORTED           # may have 2^31 key tiles
    for bad in (dict(src=P + 8), dict(dst=P + 2), dict(src_head=100), dict(src_token=4), dict(dst_head=12)):
        assert _attention(_rows(**bad), K) == ALIGNMENT, bad
    for bad in (dict(k=P + 8), dict(v=P + 4), dict(k_page=4), dict(v_head=100), dict(k_token=132)):
        assert _attention(R, _cache(**bad)) == ALIGNMENT, bad
    assert _attention(R, K, workspace=P + 128) == ALIGNMENT and _attention(R, K, lse=P + 2) == ALIGNMENT
    need = binding.efq_paged_attention_workspace_bytes(8, 2, 1)
    assert _attention(R, K, workspace=None) == WORKSPACE and _attention(R, K, nbytes=need - 1) == WORKSPACE
    assert _attention(R, K, max_q=100, nbytes=need) == WORKSPACE
    assert _attention(R, K, total=0, workspace=None) == OK and _attention(R, _cache(n_seqs=0), workspace=None) == OK       # nothing to do


def test_workspace_sizes():
    size = binding.efq_paged_attention_workspace_bytes
    assert size(8, 2, 1) == size(8, 2, 4) < size(8, 2, 5) == size(8, 2, 100000)       # 16 query rows a KV head are the line
    assert size(8, 3, 1) == 0 and size(0, 1, 1) == 0 and size(8, 2, -1) == 0 and size(8, 2, 1, 64) == 0 and size(129, 1, 1) == 0


def _rotary(q=None, k=None, positions=P, B=1, S=5, d=128, dtype=0, rotation=None):
    return binding.lib().efq_rotary(q and C.byref(q), k and C.byref(k), positions, 5, 0, B, S, d, dtype, rotation and C.byref(rotation), 0, None)


def test_rotary_refuses():
    R, T = _rows(), _rotation()
    assert _rotary(rotation=T) == INVALID and _rotary(R) == INVALID and _rotary(R, positions=None, rotation=T) == INVALID
    assert _rotary(R, B=-1, rotation=T) == INVALID and _rotary(R, S=-1, rotation=T) == INVALID
    assert _rotary(R, d=64, rotation=T) == UNSUPPORTED and _rotary(R, dtype=3, rotation=T) == UNSUPPORTED
    for bad, status in ((dict(inv_freq=None), INVALID), (dict(n_axes=0), INVALID), (dict(n_axes=5), INVALID), (dict(pairs=(C.c_int32 * 4)(-8)), INVALID),
                        (dict(pairs=(C.c_int32 * 4)(72)), UNSUPPORTED), (dict(pairs=(C.c_int32 * 4)(20)), UNSUPPORTED), (dict(inv_freq=P + 4), ALIGNMENT),
                        (dict(n_axes=2, pairs=(C.c_int32 * 4)(64, 8)), UNSUPPORTED), (dict(n_axes=2, pairs=(C.c_int32 * 4)(2**31 - 1, 65)), UNSUPPORTED)):
        assert _rotary(R, rotation=_rotation(**bad)) == status, bad
    for bad, status in ((dict(src=None), INVALID), (dict(dst=None), INVALID), (dict(heads=0), INVALID), (dict(src=P + 8), ALIGNMENT), (dict(dst_batch=4), ALIGNMENT)):
        assert _rotary(_rows(**bad), rotation=T) == status and _rotary(R, _rows(**bad), rotation=T) == status, bad
    assert _rotary(R, S=0, rotation=T) == OK and _rotary(R, B=0, rotation=T) == OK


def _append(k=None, v=None, q=None, total=5, cache=None, d=128, dtype=0, rotation=None):
    return binding.lib().efq_paged_append(k and C.byref(k), v and C.byref(v), q and C.byref(q), total, None, 0, cache and C.byref(cache), d, dtype,
                                          rotation and C.byref(rotation), None)


def test_append_refuses():
    R, K = _rows(heads=2), _cache()
    assert _append(None, R, cache=K) == INVALID and _append(R, None, cache=K) == INVALID and _append(R, R) == INVALID and _append(R, R, total=-1, cache=K) == INVALID
    assert _append(_rows(heads=3), R, cache=K) == INVALID and _append(R, _rows(heads=1), cache=K) == INVALID          # not the cache's heads
    assert _append(R, R, cache=_cache(page_size=8)) == UNSUPPORTED and _append(R, R, cache=K, dtype=-1) == UNSUPPORTED
    assert _append(R, R, cache=K, rotation=_rotation(n_axes=9)) == INVALID and _append(R, R, cache=_cache(k=P + 2)) == ALIGNMENT
    assert _append(_rows(heads=2, src=P + 8), R, cache=K) == ALIGNMENT and _append(R, R, _rows(dst=None), cache=K) == INVALID
    assert _append(R, R, total=0, cache=K) == OK and _append(R, R, cache=_cache(n_seqs=0)) == OK


@pytest.mark.gpu
def test_calls_with_tensors_do_not_hold_the_interpreter_lock(tmp_path):
    """While a call waits (here in a function that sleeps in the place of the library's), other Python threads run."""
    import subprocess
    (tmp_path / "slow.c").write_text("#include <unistd.h>\nlong slow(void) { usleep(200000); return 0; }\n")
    subprocess.run(["gcc", "-shared", "-fPIC", str(tmp_path / "slow.c"), "-o", str(tmp_path / "slow.so")], check=True)
    slow = C.cast(C.CDLL(str(tmp_path / "slow.so")).slow, C.c_void_p).value
    f = binding._tensorcall()
    make = lambda *shape, dtype=torch.bfloat16: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    cache = (make(3, 2, 16, 128), make(3, 2, 16, 128), make(1, 3, dtype=torch.int32), make(2, dtype=torch.int32), make(1, dtype=torch.int32))
    count, stop = [0], threading.Event()

    def run():
        while not stop.is_set():
            count[0] += 1
            time.sleep(0.002)

    thread = threading.Thread(target=run)
    f.set_functions(slow, slow, slow)
    thread.start()
    try:
        for call in (lambda: f.rotary(make(1, 2, 5, 128), None, make(1, 5, dtype=torch.int32), C.addressof(_rotation()), 0, make(1, 2, 5, 128), None, torch.cuda.current_device(), 0),
                     lambda: f.paged_append(make(5, 2, 128), make(5, 2, 128), *cache, None, None, None, None, torch.cuda.current_device(), 0),
                     lambda: f.paged_attention(make(5, 4, 128), *cache, 1, 1, 0.0, make(5, 4, 128), None, make(9, dtype=torch.uint8), torch.cuda.current_device(), 0)):
            before = count[0]
            assert call() == 0
            assert count[0] - before >= 5, "the other thread stood still"
    finally:
        stop.set()
        thread.join()
        binding._tensors = None
        binding._tensorcall()           # the library's own functions again


def _problem():
    g = dict(device="cuda")
    r = binding.Rotary.of((64,))
    q, k = torch.zeros(5, 4, 128, dtype=torch.bfloat16, **g), torch.zeros(5, 2, 128, dtype=torch.bfloat16, **g)
    cache = torch.zeros(3, 2, 16, 128, dtype=torch.bfloat16, **g)
    table, cu, lens = (torch.tensor(x, dtype=torch.int32, **g) for x in ([[0, 1, 2]], [0, 5], [9]))
    return r, q, k, cache, table, cu, lens


@pytest.mark.gpu
def test_the_binding_refuses():
    r, q, k, cache, table, cu, lens = _problem()
    attention = binding.efq_paged_attention_fwd
    good = [q, cache, cache.clone(), table, cu, lens, 5]
    attention(*good)
    for at, bad in ((0, q.float()), (0, q.half()), (0, q[..., :64]), (0, q.cpu()), (0, q[0]), (0, q.transpose(1, 2).contiguous().transpose(1, 2)), (0, None),
                    (1, cache[0]), (1, cache.half()), (2, cache[:2]), (2, cache.cpu()), (3, table.long()), (3, table[0]), (3, table.cpu()),
                    (4, cu[:1]), (4, cu.long()), (5, lens[:0]), (5, lens.float()), (6, -1)):
        args = list(good)
        args[at] = bad
        with pytest.raises((AssertionError, AttributeError)):
            attention(*args, workspace=torch.empty(1 << 26, dtype=torch.uint8, device="cuda"))
    for more in (dict(o=q.float()), dict(o=q[:4]), dict(lse=torch.zeros(5, 4, device="cuda").half()), dict(lse=torch.zeros(4, 5, device="cuda")),
                 dict(workspace=torch.zeros(1 << 26, device="cuda"))):
        with pytest.raises(AssertionError):
            attention(*good, **more)
    with pytest.raises(binding.EfqError) as e:
        attention(*good, workspace=torch.empty(1024, dtype=torch.uint8, device="cuda"))
    assert e.value.status == WORKSPACE
    append = binding.efq_paged_append
    good = [k, k.clone(), cache, cache.clone(), table, cu, lens, r]
    append(*good, None, q)
    for at, bad in ((0, k.half()), (0, k[:4]), (1, k[:, :1]), (1, k.cpu()), (2, cache[:, :1].contiguous()), (3, cache.half()), (4, table.long())):
        args = list(good)
        args[at] = bad
        with pytest.raises(AssertionError):
            append(*args)
    for more in (dict(q=q.half()), dict(q=q[:4]), dict(q=q, q_out=q[:4]), dict(positions=lens[None].expand(1, 5).float()), dict(positions=torch.zeros(2, 5, dtype=torch.int32, device="cuda"))):
        with pytest.raises(AssertionError):
            append(*good, **more)
    pos = torch.zeros(1, 5, dtype=torch.int32, device="cuda")
    x, y = q.transpose(0, 1)[None], k.transpose(0, 1)[None]
    binding.efq_rotary(x, y, pos, r)
    for args in ((x, y.half(), pos), (x, y[:, :, :4], pos), (x.float(), None, pos), (x, None, pos.long()), (x, None, pos[:, :4]), (x, None, pos.expand(2, 5)),
                 (None, None, pos), (x.cpu(), None, pos), (x[0], None, pos)):
        with pytest.raises(AssertionError):
            binding.efq_rotary(*args, r)
    with pytest.raises(AssertionError):
        binding.efq_rotary(x, None, pos, r, q_out=x[:, :2])
    with pytest.raises(AssertionError):
        binding.Rotary(torch.zeros(64, dtype=torch.float32, device="cuda"), (64,))
    with pytest.raises(binding.EfqError) as e:
        binding.efq_rotary(x, None, pos, binding.Rotary.of((60,)))
    assert e.value.status == UNSUPPORTED


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 40])
def test_an_expired_wait_gives_rows_of_nan(n):
    """K and V are never loaded: the waits run out, every block ends, the context stays usable."""
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(2 * n, 8, 128, generator=g, device="cuda").bfloat16()
    cache = torch.randn(40, 2, 16, 128, generator=g, device="cuda").bfloat16()
    table = torch.arange(40, dtype=torch.int32, device="cuda").view(2, 20)
    cu, lens = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda"), torch.tensor([300, 77], dtype=torch.int32, device="cuda")
    want = binding.efq_paged_attention_fwd(q, cache, cache, table, cu, lens, n)
    o = torch.zeros_like(q)
    ws = torch.empty(binding.efq_paged_attention_workspace_bytes(8, 2, n), dtype=torch.uint8, device="cuda")
    binding.efq_paged_attention_fwd_inject_timeout(q, cache, cache, table, cu, lens, n, o, ws)
    torch.cuda.synchronize()
    assert torch.isnan(o).all()
    assert torch.equal(binding.efq_paged_attention_fwd(q, cache, cache, table, cu, lens, n, o=o, workspace=ws), want)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 6, 20])
def test_an_expired_wait_in_a_step_of_many_sequences(n):
    """Blocks have many query tiles to go when the first wait runs out: all their rows become NaN, those without a key are zeros as ever."""
    seqs = 400
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(seqs * n, 8, 128, generator=g, device="cuda").bfloat16()
    cache = torch.randn(64, 2, 16, 128, generator=g, device="cuda").bfloat16()
    table = torch.randint(0, 64, (seqs, 12), generator=g, dtype=torch.int32, device="cuda")
    cu = torch.arange(0, seqs * n + 1, n, dtype=torch.int32, device="cuda")
    lens = torch.tensor([0 if i % 7 == 3 else n + (i * 11) % 170 for i in range(seqs)], dtype=torch.int32, device="cuda")
    want = binding.efq_paged_attention_fwd(q, cache, cache, table, cu, lens, n)
    o = torch.zeros_like(q)
    ws = torch.empty(binding.efq_paged_attention_workspace_bytes(8, 2, n), dtype=torch.uint8, device="cuda")
    binding.efq_paged_attention_fwd_inject_timeout(q, cache, cache, table, cu, lens, n, o, ws)
    torch.cuda.synchronize()
    seen = (lens > 0).repeat_interleave(n)
    assert torch.isnan(o[seen]).all() and (torch.isnan(o[~seen]) | (o[~seen] == 0)).all()
    assert torch.equal(binding.efq_paged_attention_fwd(q, cache, cache, table, cu, lens, n, o=o, workspace=ws), want)


def test_tables_and_positions_on_odd_addresses_are_refused():
    """32-bit loads from an address that is no multiple of four fault."""
    T = _rotation()
    for name in ("page_table", "cu_seqlens", "seq_lens"):
        bad = _cache(**{name: P + 2})
        assert _attention(_rows(), bad) == ALIGNMENT and _append(_rows(heads=2), _rows(heads=2), cache=bad, rotation=T) == ALIGNMENT, name
    assert _rotary(_rows(), positions=P + 2, rotation=T) == ALIGNMENT
    R, K = _rows(heads=2), _cache()
    assert binding.lib().efq_paged_append(C.byref(R), C.byref(R), None, 5, P + 1, 5, C.byref(K), 128, 0, C.byref(T), None) == ALIGNMENT


def test_more_heads_than_32_bits_are_refused():
    most = 2**31 - 1
    assert _rotary(_rows(heads=most), _rows(heads=most), rotation=_rotation()) == UNSUPPORTED
    assert _append(_rows(heads=2), _rows(heads=2), _rows(heads=most), cache=_cache()) == UNSUPPORTED


@pytest.mark.parametrize("page", [16, 32, 64, 128, 4096])
def test_tokens_of_a_sequence_end_a_tile_before_31_bits(page):
    """The kernels' keys are 32-bit numbers up to the end of the last tile of 128: a page table with room for more than 2^31 - 256 tokens is refused."""
    most = (2**31 - 256) // page
    for max_pages in (2**31 // page - 1, most + 1):
        if max_pages * page > 2**31 - 256:
            bad = _cache(page_size=page, max_pages=max_pages, n_seqs=1)
            assert _attention(_rows(), bad) == UNSUPPORTED and _append(_rows(heads=2), _rows(heads=2), cache=bad) == UNSUPPORTED, max_pages
    good = _cache(page_size=page, max_pages=most, n_seqs=0)
    assert _attention(_rows(), good) == OK and _append(_rows(heads=2), _rows(heads=2), cache=good) == OK


@pytest.mark.parametrize("heads", [2**24, 2**25, 2**27 + 3, 2**30, 2**31 - 1])
def test_steps_of_more_key_tiles_than_31_bits_are_refused_for_any_number_of_heads(heads):
    """Sequences times tiles of a context times heads are 2^63 and more here."""
    for n_seqs in (40000 * 2**24 // heads, 50000 * 2**24 // heads, 65000 * 2**24 // heads):
        assert _attention(_rows(heads=heads), _cache(n_heads=heads, max_pages=2**26, n_seqs=n_seqs), total=1) == UNSUPPORTED, n_seqs


def test_scales_that_are_infinite_in_units_of_log2_are_refused():
    for scale in (2.4e38, 3.0e38, 3.4e38):
        assert _attention(_rows(), _cache(), scale=scale) == INVALID, scale
    for scale in (2.3e38, 1e-45, -1.0, float("-inf")):
        assert _attention(_rows(), _cache(), scale=scale, total=0) == OK, scale


@pytest.mark.gpu
@pytest.mark.parametrize("n,seqs", [(1, 2), (6, 2), (40, 2), (1, 300), (7, 90)])
def test_the_status_of_a_call_is_in_its_workspace(n, seqs):
    """0 after a call, whatever stood there; the time-out after one whose waits expired; 0 again after the next."""
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randn(seqs * n, 8, 128, generator=g, device="cuda").bfloat16()
    cache = torch.randn(40, 2, 16, 128, generator=g, device="cuda").bfloat16()
    table = torch.randint(0, 40, (seqs, 20), generator=g, dtype=torch.int32, device="cuda")
    cu = torch.arange(0, seqs * n + 1, n, dtype=torch.int32, device="cuda")
    lens = torch.tensor([n + (i * 37 + 250) % 260 for i in range(seqs)], dtype=torch.int32, device="cuda")
    nbytes = binding.efq_paged_attention_workspace_bytes(8, 2, n)
    guard = torch.full((nbytes + 4096,), 255, dtype=torch.uint8, device="cuda")
    ws, o, side = guard[:nbytes], torch.empty_like(q), torch.cuda.Stream()
    args = (q, cache, cache, table, cu, lens, n)
    for _ in range(2):
        binding.efq_paged_attention_fwd(*args, o=o, workspace=ws)
        assert binding.efq_poll_status(ws) == OK
        binding.efq_paged_attention_fwd_inject_timeout(*args, o, ws)
        assert binding.efq_poll_status(ws) == binding.STATUS_NAMES.index("EFQ_ERR_DEVICE_TIMEOUT")
    torch.cuda.synchronize()
    binding.efq_paged_attention_fwd(*args, o=o, workspace=ws, stream=side)
    assert binding.efq_poll_status(ws, side) == OK and torch.isfinite(o).all()
    assert (guard[nbytes:] == 255).all()
