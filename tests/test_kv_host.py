"""Cache, attention, residual norm without a GPU: sizes, and every refusal before any CUDA call (the pointers are fakes that
are never followed)."""
import ctypes

import pytest

import paper_2402_15319_b200 as vq
from paper_2402_15319_b200 import binding, build as vq_build
from tests.kv_ref import Books

FAKE, ODD, ODD4 = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008), ctypes.c_void_p(0x10002)
GOOD = vq.VQKVFormat(32, 16, 4, 128, vq.VQ_KV_FP16)
OK, NULL, FORMAT, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 5, 7


@pytest.fixture(scope="module", autouse=True)
def _built():
    vq_build.build()


def _fmt(**kw):
    return vq.VQKVFormat(**{**GOOD.__dict__, **kw})


def _pool(fmt, **kw):
    i8 = fmt.kv_type == vq.VQ_KV_INT8
    f = dict(d_k=FAKE, d_v=FAKE, d_k_scale=FAKE if i8 else None, d_v_scale=FAKE if i8 else None)
    return binding._CKVPool(**{**f, **kw})


def _seqs(**kw):
    return binding._CKVSeqs(**{**dict(d_table=FAKE, d_len=FAKE, n_seqs=3, table_stride=8), **kw})


def test_sizes():
    i = vq.vq_kv_info(GOOD)
    assert i.pool_bytes == 32 * 4 * 16 * 128 * 2 and i.scale_bytes == 0 and i.page_bytes == 2 * 4 * 16 * 256
    i = vq.vq_kv_info(_fmt(kv_type=vq.VQ_KV_INT8, head_dim=80))
    assert i.pool_bytes == 32 * 4 * 16 * 80 and i.scale_bytes == 32 * 4 * 16 * 4 and i.page_bytes == 2 * 4 * 16 * 84
    assert vq.vq_kv_info(_fmt(n_pages=1 << 20)).pool_bytes == (1 << 20) * 4 * 16 * 256   # beyond 32 bits
    assert vq.vq_kv_attention_workspace_bytes(GOOD) > 0
    assert vq.vq_kv_attention_workspace_bytes(_fmt(head_dim=48)) == 0     # no kernel for it
    assert vq.vq_kv_pages_workspace_bytes(GOOD, 5) > 0 and vq.vq_kv_pages_workspace_bytes(GOOD, 0) == 0
    assert vq.vq_kv_pages_workspace_bytes(_fmt(n_pages=100), 7) > vq.vq_kv_pages_workspace_bytes(_fmt(n_pages=10), 7)


@pytest.mark.parametrize("kw,code", [
    (dict(kv_type=2), FORMAT), (dict(kv_type=-1), FORMAT), (dict(page_tokens=4), FORMAT), (dict(page_tokens=24), FORMAT), (dict(page_tokens=512), FORMAT),
    (dict(page_tokens=0), FORMAT), (dict(head_dim=0), FORMAT), (dict(head_dim=72), FORMAT), (dict(head_dim=272), FORMAT), (dict(head_dim=-16), FORMAT),
    (dict(n_pages=0), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(n_kv_heads=-3), SHAPE),
])
def test_bad_formats(kw, code):
    f = _fmt(**kw)
    with pytest.raises(vq.VQError) as e:
        vq.vq_kv_info(f)
    assert e.value.code == code
    assert vq.vq_kv_attention_workspace_bytes(f) == 0 and vq.vq_kv_pages_workspace_bytes(f, 3) == 0
    assert _attend(f) == code and _append(f) == code and _reserve(f) == code and _fork(f) == code and _compact(f) == code
    assert _free(f) == code and _copy(f) == code


def _attend(fmt=GOOD, pool=None, seqs=None, hq=8, q=FAKE, qs=1024, out=FAKE, os=1024, lse=None, window=0, ws=FAKE, ws_bytes=1 << 30):
    pool, seqs, c = pool or _pool(fmt), seqs or _seqs(), fmt.c()
    return vq.load().vq_kv_attention(ctypes.byref(c), ctypes.byref(pool), ctypes.byref(seqs), hq, q, qs, out, os, lse, 0.1, window, ws, ws_bytes, None)


def test_attention_refusals():
    i8 = _fmt(kv_type=vq.VQ_KV_INT8)
    for kw in (dict(d_k=None), dict(d_v=None), dict(d_k_scale=FAKE), dict(d_v_scale=FAKE)):
        assert _attend(pool=_pool(GOOD, **kw)) == NULL
    assert _attend(i8, pool=_pool(i8, d_k_scale=None)) == NULL
    assert _attend(pool=_pool(GOOD, d_k=ODD)) == ALIGN and _attend(i8, pool=_pool(i8, d_v_scale=ODD)) == ALIGN
    assert _attend(seqs=_seqs(d_table=None)) == NULL and _attend(seqs=_seqs(d_len=None)) == NULL
    assert _attend(seqs=_seqs(d_len=ODD4)) == ALIGN
    for kw in (dict(n_seqs=0), dict(n_seqs=65537), dict(table_stride=0), dict(table_stride=-1), dict(table_stride=(1 << 26) + 1)):
        assert _attend(seqs=_seqs(**kw)) == SHAPE
    assert _attend(q=None) == NULL and _attend(out=None) == NULL
    assert _attend(q=ODD) == ALIGN and _attend(out=ODD) == ALIGN and _attend(lse=ODD4) == ALIGN and _attend(ws=ODD) == ALIGN
    assert _attend(hq=0) == SHAPE and _attend(hq=6) == SHAPE and _attend(hq=-4) == SHAPE and _attend(window=-1) == SHAPE
    assert _attend(qs=1023) == SHAPE and _attend(os=1000) == SHAPE and _attend(qs=1028) == ALIGN and _attend(os=1025) == ALIGN
    assert _attend(ws=None) == WORKSPACE and _attend(ws_bytes=vq.vq_kv_attention_workspace_bytes(GOOD) - 1) == WORKSPACE
    assert _attend(_fmt(head_dim=48)) == UNSUPPORTED


def _append(fmt=GOOD, pool=None, seqs=None, starts=None, n=3, k=FAKE, ks=512, v=FAKE, vs=512, rot=None):
    pool, seqs, c = pool or _pool(fmt), seqs or _seqs(), fmt.c()
    return vq.load().vq_kv_append(ctypes.byref(c), ctypes.byref(pool), ctypes.byref(seqs), starts, n, k, ks, v, vs,
                                  None if rot is None else ctypes.byref(rot), None)


def _rot(**kw):
    f = dict(d_cos_sin=FAKE, n_positions=128, rot_dim=128, interleaved=0, n_q_heads=8, d_q=FAKE, d_q_out=FAKE, q_stride=1024, q_out_stride=1024)
    return binding._CKVRotary(**{**f, **kw})


def test_append_refusals():
    assert _append(k=None) == NULL and _append(v=None) == NULL and _append(pool=_pool(GOOD, d_v=None)) == NULL
    assert _append(n=2) == SHAPE and _append(n=0, starts=FAKE) == SHAPE and _append(ks=511) == SHAPE and _append(vs=500) == SHAPE
    assert _append(ks=516) == ALIGN and _append(k=ODD) == ALIGN and _append(v=ODD) == ALIGN and _append(starts=ODD4) == ALIGN
    assert _append(rot=_rot(d_cos_sin=None)) == NULL and _append(rot=_rot(d_q=None)) == NULL and _append(rot=_rot(d_q_out=None)) == NULL
    assert _append(rot=_rot(n_q_heads=0)) == NULL         # queries without heads
    for kw in (dict(rot_dim=8), dict(rot_dim=144), dict(rot_dim=24), dict(n_q_heads=-1), dict(n_positions=127), dict(interleaved=2), dict(q_stride=1016),
               dict(q_out_stride=8), dict(q_stride=1032)):
        assert _append(rot=_rot(**kw)) == SHAPE, kw       # (the last: in place, with another stride)
    assert _append(rot=_rot(d_cos_sin=ODD)) == ALIGN and _append(rot=_rot(d_q=ODD)) == ALIGN and _append(rot=_rot(q_stride=1028)) == ALIGN


def _reserve(fmt=GOOD, seqs=None, refs=FAKE, new=None, status=FAKE, ws=FAKE, ws_bytes=1 << 30):
    seqs, c = seqs or _seqs(), fmt.c()
    return vq.load().vq_kv_reserve(ctypes.byref(c), ctypes.byref(seqs), refs, new, status, ws, ws_bytes, None)


def _fork(fmt=GOOD, n_layers=2, seqs=None, refs=FAKE, pairs=FAKE, n=2, status=FAKE, ws=FAKE, ws_bytes=1 << 30, pools=True):
    seqs, c = seqs or _seqs(), fmt.c()
    arr = (binding._CKVPool * 121)(*[_pool(fmt)] * 121) if pools else None
    return vq.load().vq_kv_fork(ctypes.byref(c), arr, n_layers, ctypes.byref(seqs), refs, pairs, n, status, ws, ws_bytes, None)


def _compact(fmt=GOOD, n_layers=2, seqs=None, refs=FAKE, status=FAKE, ws=FAKE, ws_bytes=1 << 30, pools=True):
    seqs, c = seqs or _seqs(), fmt.c()
    arr = (binding._CKVPool * 121)(*[_pool(fmt)] * 121) if pools else None
    return vq.load().vq_kv_compact(ctypes.byref(c), arr, n_layers, ctypes.byref(seqs), refs, status, ws, ws_bytes, None)


def _copy(fmt=GOOD, n_layers=2, pairs=FAKE, n=2, pools=True):
    c = fmt.c()
    arr = (binding._CKVPool * 121)(*[_pool(fmt)] * 121) if pools else None
    return vq.load().vq_kv_copy_pages(ctypes.byref(c), arr, n_layers, pairs, n, None)


def _free(fmt=GOOD, seqs=None, refs=FAKE, slots=FAKE, n=2):
    seqs, c = seqs or _seqs(), fmt.c()
    return vq.load().vq_kv_free(ctypes.byref(c), ctypes.byref(seqs), refs, slots, n, None)


def test_page_refusals():
    need = vq.vq_kv_pages_workspace_bytes(GOOD, 3)
    for call in (_reserve, _fork, _compact):
        assert call(refs=None) == NULL and call(status=None) == NULL and call(refs=ODD4) == ALIGN and call(status=ODD4) == ALIGN
        assert call(ws=None) == WORKSPACE and call(ws_bytes=need - 1) == WORKSPACE and call(ws=ODD) == ALIGN
        assert call(seqs=_seqs(n_seqs=0)) == SHAPE and call(seqs=_seqs(d_len=None)) == NULL
    assert _reserve(new=ODD4) == ALIGN
    for call in (_fork, _compact, _copy):
        assert call(pools=False) == NULL and call(n_layers=0) == SHAPE and call(n_layers=121) == SHAPE
    assert _fork(pairs=None) == NULL and _fork(n=0) == SHAPE and _fork(n=1025) == SHAPE and _fork(pairs=ODD4) == ALIGN
    assert _copy(pairs=None) == NULL and _copy(n=0) == SHAPE and _copy(n=(1 << 24) + 1) == SHAPE and _copy(pairs=ODD4) == ALIGN
    assert _free(slots=None) == NULL and _free(refs=None) == NULL and _free(n=0) == SHAPE and _free(n=65537) == SHAPE and _free(slots=ODD4) == ALIGN


NORM = vq.VQNorm(4, 64, vq.VQ_NORM_RMS, vq.VQ_RESIDUAL_FP16, vq.VQ_GATE_NONE, 1e-5, 1.0, 64, 64, 64, 64, 64)


def _norm(x=FAKE, y=FAKE, gate=None, post_w=None, post_b=None, pre_w=FAKE, pre_b=None, x_out=FAKE, h=FAKE, **kw):
    c = vq.VQNorm(**{**NORM.__dict__, **kw}).c()
    return vq.load().vq_residual_norm(ctypes.byref(c), x, y, gate, post_w, post_b, pre_w, pre_b, x_out, h, None)


def test_norm_refusals():
    other = ctypes.c_void_p(0x20000)
    assert vq.load().vq_residual_norm(None, *[FAKE] * 9, None) == NULL
    assert _norm(x=None) == NULL and _norm(x_out=None, h=None, pre_w=None) == NULL
    assert _norm(pre_w=None) == NULL and _norm(h=None) == NULL                # a norm and its output come together
    assert _norm(gate=FAKE) == NULL                                           # a gate that the block does not name
    assert _norm(post_b=FAKE) == NULL and _norm(h=None, pre_w=None, pre_b=FAKE) == NULL
    assert _norm(y=None, post_w=FAKE) == NULL and _norm(y=None, post_w=FAKE, post_b=FAKE) == NULL
    c = vq.VQNorm(**{**NORM.__dict__, "gate": vq.VQ_GATE_CHANNEL}).c()
    assert vq.load().vq_residual_norm(ctypes.byref(c), FAKE, FAKE, None, None, None, FAKE, None, FAKE, other, None) == NULL
    for kw in (dict(kind=2), dict(kind=-1), dict(residual_type=2)):
        assert _norm(**kw) == FORMAT
    c = vq.VQNorm(**{**NORM.__dict__, "gate": 3}).c()
    assert vq.load().vq_residual_norm(ctypes.byref(c), FAKE, FAKE, FAKE, None, None, FAKE, None, FAKE, other, None) == FORMAT
    for kw in (dict(n_rows=0), dict(n_cols=0), dict(n_cols=32769), dict(n_cols=65), dict(x_stride=63), dict(y_stride=63), dict(x_out_stride=63),
               dict(h_stride=63)):
        assert _norm(h=other, **kw) == SHAPE, kw
    assert _norm(h=other, x_out_stride=72) == SHAPE and _norm(h=FAKE, h_stride=72, x_out=other) == SHAPE   # in place with another stride
    for name in ("x", "y", "pre_w", "x_out", "h", "pre_b"):
        assert _norm(**{"h": other, **{name: ODD}}) == ALIGN
    assert _norm(h=other, post_w=ODD) == ALIGN


def test_host_tensors_are_refused():
    torch = pytest.importorskip("torch")
    t = torch.zeros(8, 8, dtype=torch.int32)
    with pytest.raises(ValueError, match="current device"):
        vq.vq_kv_reserve(GOOD, vq.KVSeqs(t, t[0].contiguous()), t, None, t, t)
    with pytest.raises(ValueError, match="current device"):
        vq.vq_residual_norm(NORM, t, t, None, None, None, t, None, t, t)


def test_handles_check_their_tensors():
    torch = pytest.importorskip("torch")
    half, i8, f32, i32 = (torch.zeros(64, dtype=t) for t in (torch.float16, torch.int8, torch.float32, torch.int32))
    for bad in ((f32, f32), (half, i8), (i8, i8), (i8, i8, half, half), (half, half, f32, f32), (half[::2], half[::2])):
        with pytest.raises(ValueError, match="KVPool"):
            vq.KVPool(*bad)
    for bad in ((i32.long().view(8, 8), i32[:8]), (i32.view(8, 8), f32[:8]), (i32.view(8, 8), i32[:7]), (i32.view(8, 8)[:, 2:], i32[:8]), (i32, i32)):
        with pytest.raises(ValueError, match="KVSeqs"):
            vq.KVSeqs(*bad)
    with pytest.raises(ValueError, match="KVRotary"):
        vq.KVRotary(f32, 5, 16, 0)
    with pytest.raises(ValueError, match="KVRotary"):
        vq.KVRotary(half, 4, 16, 0)
    small = vq.VQKVFormat(2, 8, 1, 16, vq.VQ_KV_FP16)
    full, short, bytes_ = (torch.zeros(n, dtype=t) for n, t in ((256, torch.float16), (255, torch.float16), (256, torch.int8)))
    binding._room(vq.KVPool(full, full), small)
    for k, v, ks, vs in ((short, full, None, None), (full, short, None, None), (bytes_, bytes_, f32[:15], f32[:16])):
        with pytest.raises(ValueError, match="smaller"):
            binding._room(vq.KVPool(k, v, ks, vs), small)


def test_handles_copied():
    """A copy's struct is its own: its address outlives the original."""
    import copy
    import pickle
    for h in (GOOD, NORM):
        for c in (copy.copy(h), copy.deepcopy(h), pickle.loads(pickle.dumps(h))):
            assert c == h and hash(c) == hash(h) and c._p == ctypes.addressof(c._c) and c._p != h._p
            assert bytes(c._c) == bytes(h._c)


def test_books_follow_the_rules():
    """The model that the GPU tests compare with, on a case worked out by hand."""
    b = Books(8, 8, 4, 4)
    assert b.reserve([17, 0, 8, 0]) == (0, 0)
    assert b.table[0][:3] == [0, 1, 2] and b.table[2][:1] == [3] and b.len == [17, 0, 8, 0]
    assert b.reserve([0, 0, 0, 33]) == (0, 1)                    # five pages, a row has four
    assert b.reserve([9, 30, 0, 0]) == (1, 0)                    # 1 + 4 pages, four are free
    status, copies = b.fork([(0, 1), (0, 1), (2, 3), (9, 3), (0, 2)])
    assert status == (0, 3) and copies == [(2, 4, 1)]            # page 2 has one token
    assert b.table[1][:3] == [0, 1, 4] and b.table[3][0] == 3 and b.refs == [2, 2, 1, 2, 1, 0, 0, 0] and b.len == [17, 17, 8, 8]
    b.free([0, 0, 7])
    assert b.refs == [1, 1, 0, 2, 1, 0, 0, 0] and b.len[0] == 0
    status, copies = b.compact()
    assert status == (4, 1) and copies == [(4, 2, 8)] and b.table[1][:3] == [0, 1, 2] and b.refs == [1, 1, 1, 2, 0, 0, 0, 0]


def test_remote_stores_wait_for_the_cluster():
    """A CTA's shared memory may be written by another one of the cluster only after it is known to have started.  Read in the
    source: each cluster kernel of the books arrives before anything else, and whoever stores has waited in front, in every span."""
    import os
    import re
    src = open(os.path.join(vq_build.CSRC, "vq_kv_pages.cu")).read()
    src = re.sub(r"//[^\n]*", "", src)

    def body(at):
        at = depth = src.index("{", at) + 1
        level = 1
        while level:
            level += {"{": 1, "}": -1}.get(src[depth], 0)
            depth += 1
        return src[at:depth]

    kernels = [m.end() for m in re.finditer(r"__cluster_dims__[^;{]*?\w+_kernel\(", src)]
    assert len(kernels) == 3
    for k in kernels:
        b = body(k)
        assert 0 <= b.find("cluster_arrive") < min(i for i in (b.find("page_bits("), b.find("free_pages("), b.find("return")) if i >= 0)
        assert b.find("cluster_wait") < 0 and b.count("cluster_arrive") == 1      # (its wait is page_bits')
    stores = [m.start() for m in re.finditer(r"st_cluster_u32\(dst", src)]
    bits = body(src.index("PageBits page_bits("))
    assert len(stores) == 1 and bits.count("st_cluster_u32(") == 1                # nothing else of the file stores remotely
    order = [bits.index("cluster_wait"), bits.index("st_cluster_u32("), bits.index("cluster_arrive"), bits.rindex("cluster_wait")]
    assert order == sorted(order) and bits.count("cluster_wait") == 2 and bits.count("cluster_arrive") == 1
    span = body(src.index("void next_span("))
    assert "cluster_arrive" in span and "cluster_wait" not in span                # the next page_bits waits for it


@pytest.mark.parametrize("dim,kv_type,heads,tokens", [
    (128, vq.VQ_KV_FP16, 1, 1 << 25), (80, vq.VQ_KV_FP16, 4, 1 << 25), (64, vq.VQ_KV_FP16, 1, 1 << 26), (256, vq.VQ_KV_INT8, 2, 1 << 25),
    (128, vq.VQ_KV_INT8, 1, 1 << 26), (64, vq.VQ_KV_INT8, 1, 1 << 27),
])
def test_attention_rows_too_long_to_number(dim, kv_type, heads, tokens):
    """The first row length behind 2^21 tiles is refused, before any CUDA call (that the last one is taken: test_gpu_kv.py)."""
    fmt = _fmt(page_tokens=256, n_kv_heads=heads, head_dim=dim, kv_type=kv_type)
    kw = dict(hq=heads, qs=heads * dim, os=heads * dim)
    assert _attend(fmt, seqs=_seqs(table_stride=tokens // 256 + 1), **kw) == UNSUPPORTED
    assert _attend(fmt, seqs=_seqs(table_stride=1 << 22), window=tokens, **kw) == UNSUPPORTED     # (and a tile that it begins inside)


def test_attention_too_much_to_number():
    wide = _fmt(page_tokens=256, n_kv_heads=512, head_dim=128)
    kw = dict(hq=512, qs=512 * 128, os=512 * 128)
    assert _attend(wide, seqs=_seqs(table_stride=131072), **kw) == UNSUPPORTED                     # (2^21 + 2) * 512 places of a sequence
    assert _attend(_fmt(n_pages=1 << 30, page_tokens=8, n_kv_heads=1), hq=1, qs=128, os=128) == UNSUPPORTED    # 2^33 rows of keys


def _on_device(monkeypatch):
    """Host tensors pass as the current device's, and no call gets as far as the library."""
    monkeypatch.setattr(binding, "_device_now", lambda: -1)
    monkeypatch.setattr(binding, "load", lambda: pytest.fail("the call went to the library"))
    monkeypatch.setattr(binding, "_stream", lambda stream: 0)


def test_books_check_their_lists(monkeypatch):
    """Page lists, counts and statuses are contiguous int32 of the lengths that the calls read."""
    torch = pytest.importorskip("torch")
    _on_device(monkeypatch)
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    fmt = vq.VQKVFormat(6, 8, 1, 16, vq.VQ_KV_FP16)
    seqs, ws = vq.KVSeqs(ints(3, 2), ints(3)), torch.zeros(1 << 16, dtype=torch.uint8)
    half = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    pools = [vq.KVPool(half(6, 1, 8, 16), half(6, 1, 8, 16))]
    good = dict(refs=ints(6), new=ints(3), status=ints(2), pairs=ints(4, 2), slots=ints(4), starts=ints(4))
    calls = {
        "reserve": (lambda a: vq.vq_kv_reserve(fmt, seqs, a["refs"], a["new"], a["status"], ws), ("refs", "new", "status")),
        "fork": (lambda a: vq.vq_kv_fork(fmt, pools, seqs, a["refs"], a["pairs"], 4, a["status"], ws), ("refs", "pairs", "status")),
        "free": (lambda a: vq.vq_kv_free(fmt, seqs, a["refs"], a["slots"], 4), ("refs", "slots")),
        "compact": (lambda a: vq.vq_kv_compact(fmt, pools, seqs, a["refs"], a["status"], ws), ("refs", "status")),
        "copy_pages": (lambda a: vq.vq_kv_copy_pages(fmt, pools, a["pairs"], 4), ("pairs",)),
        "append": (lambda a: vq.vq_kv_append(fmt, pools[0], seqs, a["starts"], 5, half(5, 16), 16, half(5, 16), 16), ("starts",)),
    }
    for name, (call, used) in calls.items():
        for key in used:
            t = good[key]
            for bad in (t.long(), t.float(), torch.zeros(2 * t.numel(), dtype=torch.int32)[::2], t.reshape(-1)[:-1].clone(), t.reshape(-1)[:0]):
                with pytest.raises(ValueError, match="int32"):
                    call({**good, key: bad})
        with pytest.raises(pytest.fail.Exception, match="library"):       # the good ones go through
            call(good)
    with pytest.raises(pytest.fail.Exception, match="library"):           # one token each: no counts
        calls["reserve"][0]({**good, "new": None})


def test_operands_of_another_type_are_refused(monkeypatch):
    """bfloat16 has binary16's size: read as it, it would give numbers, and wrong ones."""
    torch = pytest.importorskip("torch")
    _on_device(monkeypatch)
    half = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    f32 = lambda *s: torch.zeros(s, dtype=torch.float32)  # noqa: E731
    ints = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    fmt = vq.VQKVFormat(6, 8, 1, 64, vq.VQ_KV_FP16)
    pool, seqs, ws = vq.KVPool(half(6, 1, 8, 64), half(6, 1, 8, 64)), vq.KVSeqs(ints(3, 2), ints(3)), torch.zeros(1 << 16, dtype=torch.uint8)
    norm = vq.VQNorm(4, 64, vq.VQ_NORM_LAYER, vq.VQ_RESIDUAL_FP16, vq.VQ_GATE_ELEMENT, 1e-5, 1.0, 64, 64, 64, 64, 64)
    wide = vq.VQNorm(**{**norm.__dict__, "residual_type": vq.VQ_RESIDUAL_FP32})
    rows, line = half(4, 64), half(64)
    calls = [
        (lambda q, out, lse: vq.vq_kv_attention(fmt, pool, seqs, 1, q, 64, out, 64, lse, 0.1, 0, ws), (half(3, 64), half(3, 64), f32(3, 1))),
        (lambda k, v: vq.vq_kv_append(fmt, pool, seqs, None, 3, k, 64, v, 64), (half(3, 64), half(3, 64))),
        (lambda *t: vq.vq_residual_norm(norm, *t), (rows, rows, rows, line, line, line, line, rows, rows)),
        (lambda *t: vq.vq_residual_norm(wide, *t), (f32(4, 64), rows, rows, line, line, line, line, f32(4, 64), rows)),
    ]
    for call, good in calls:
        for i, t in enumerate(good):
            for other in (torch.bfloat16, torch.float32 if t.dtype == torch.float16 else torch.float16, torch.int16):
                with pytest.raises(ValueError, match="float"):
                    call(*good[:i], t.to(other), *good[i + 1:])
        with pytest.raises(pytest.fail.Exception, match="library"):
            call(*good)
    with pytest.raises(pytest.fail.Exception, match="library"):           # absent operands
        vq.vq_residual_norm(norm, rows, None, None, None, None, line, None, None, rows)
    for q, out in ((rows.bfloat16(), rows), (rows, f32(4, 64))):
        with pytest.raises(ValueError, match="float"):
            vq.KVRotary(f32(16, 32, 2), 16, 64, 0, 1, q, 64, out, 64)
