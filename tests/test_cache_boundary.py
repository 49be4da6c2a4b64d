"""Refusals of the calls around the paged cache: on the host, before anything is launched, so they run without a GPU."""
import ctypes

import pytest

import paper_2505_19578_amd as sp

FAKE = 4096  # an address that is never looked at: every call here is refused first


def _cache(**kw):
    c = sp.SpCacheShape()
    c.n_pages, c.page_size, c.n_kv_heads, c.head_dim = 8, 16, 2, 64
    c.stride_page, c.stride_token, c.stride_head = 16 * 128, 128, 64
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _step(**kw):
    s = sp.SpStepShape()
    s.n_requests, s.n_tokens, s.n_q_heads, s.max_new, s.max_pages, s.mask_words = 2, 6, 4, 3, 4, 1
    s.q_stride_t, s.q_stride_h, s.o_stride_t, s.o_stride_h = 256, 64, 256, 64
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _rope(**kw):
    s = sp.SpRopeShape()
    s.n_tokens, s.n_q_heads, s.n_kv_heads, s.head_dim, s.rotary_dim, s.eps = 5, 4, 2, 64, 64, 1e-6
    for x, h in (("q", 4), ("k", 2), ("v", 2), ("qo", 4), ("ko", 2)):
        setattr(s, x + "_stride_t", 64 * h)
        setattr(s, x + "_stride_h", 64)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _said(rc, status, text=b""):
    L = sp.lib()
    assert L.sp_status_string(rc) == status.encode(), (L.sp_status_string(rc), L.sp_last_error())
    assert text in L.sp_last_error(), L.sp_last_error()


BAD_CACHES = [
    (dict(n_pages=0), "SP_ERR_INVALID_ARG", b"n_pages"), (dict(page_size=8), "SP_ERR_UNSUPPORTED", b"page_size"),
    (dict(page_size=48), "SP_ERR_UNSUPPORTED", b"page_size"), (dict(page_size=8192), "SP_ERR_UNSUPPORTED", b"page_size"),
    (dict(page_size=-16), "SP_ERR_UNSUPPORTED", b"page_size"), (dict(head_dim=96), "SP_ERR_UNSUPPORTED", b"head_dim"),
    (dict(n_kv_heads=0), "SP_ERR_INVALID_ARG", b"head counts"), (dict(stride_token=132), "SP_ERR_INVALID_ARG", b"stride_token"),
    (dict(stride_token=56), "SP_ERR_INVALID_ARG", b"stride_token"), (dict(stride_page=-8), "SP_ERR_INVALID_ARG", b"stride_page"),
    (dict(stride_token=(1 << 24) + 8), "SP_ERR_UNSUPPORTED", b"stride_token"),
    (dict(n_pages=1 << 27), "SP_ERR_UNSUPPORTED", b"slots"),
]


@pytest.mark.parametrize("bad,status,text", BAD_CACHES)
def test_cache_geometry(bad, status, text):
    L, n = sp.lib(), ctypes.c_size_t(0)
    _said(L.sp_cache_attn_workspace_bytes(ctypes.byref(_step()), ctypes.byref(_cache(**bad)), ctypes.byref(n)), status, text)
    c = _cache(**bad)
    rc = L.sp_cache_accept(ctypes.byref(c), 1, 0, FAKE, FAKE, 1, 4, FAKE, FAKE, FAKE, 4, FAKE, FAKE, None, None)
    _said(rc, status, text)
    rc = L.sp_qk_norm_rope(ctypes.byref(_rope()), *[FAKE] * 9, ctypes.byref(c), FAKE, FAKE, FAKE, None)
    _said(rc, status, text)


@pytest.mark.parametrize("bad,status,text", [
    (dict(n_requests=-1), "SP_ERR_INVALID_ARG", b"negative"), (dict(n_tokens=-1), "SP_ERR_INVALID_ARG", b"negative"),
    (dict(n_requests=(1 << 20) + 1), "SP_ERR_UNSUPPORTED", b"2^20"), (dict(n_tokens=(1 << 28) + 1), "SP_ERR_UNSUPPORTED", b"2^28"),
    (dict(max_pages=0), "SP_ERR_INVALID_ARG", b"max_pages"), (dict(max_new=0), "SP_ERR_INVALID_ARG", b"max_new"),
    (dict(mask_words=5), "SP_ERR_UNSUPPORTED", b"mask_words"), (dict(mask_words=-1), "SP_ERR_UNSUPPORTED", b"mask_words"),
    (dict(max_new=65), "SP_ERR_INVALID_ARG", b"max_new"), (dict(n_q_heads=3), "SP_ERR_INVALID_ARG", b"n_q_heads"),
    (dict(n_q_heads=2048), "SP_ERR_UNSUPPORTED", b"n_q_heads"), (dict(max_pages=1 << 27), "SP_ERR_UNSUPPORTED", b"longer"),
    (dict(q_stride_t=260), "SP_ERR_INVALID_ARG", b"q_stride_t"), (dict(q_stride_h=32), "SP_ERR_INVALID_ARG", b"q_stride_h"),
    (dict(o_stride_t=-8), "SP_ERR_INVALID_ARG", b"o_stride_t"), (dict(o_stride_h=60), "SP_ERR_INVALID_ARG", b"o_stride_h"),
    (dict(softmax_scale=-1.0), "SP_ERR_INVALID_ARG", b"softmax_scale"),
    (dict(softmax_scale=float("nan")), "SP_ERR_INVALID_ARG", b"softmax_scale"),
    (dict(softmax_scale=float("inf")), "SP_ERR_INVALID_ARG", b"softmax_scale"),
    (dict(n_requests=1 << 20, n_tokens=1 << 28, max_pages=1 << 22, mask_words=0), "SP_ERR_UNSUPPORTED", b"too large"),
])
def test_attention_geometry(bad, status, text):
    L, n = sp.lib(), ctypes.c_size_t(0)
    _said(L.sp_cache_attn_workspace_bytes(ctypes.byref(_step(**bad)), ctypes.byref(_cache()), ctypes.byref(n)), status, text)


def test_attention_arguments():
    L, s, c = sp.lib(), _step(max_pages=400), _cache()
    bytes_needed = sp.sp_cache_attn_workspace_bytes(s, c)
    assert bytes_needed > 0 and sp.sp_cache_attn_workspace_bytes(_step(), c) == 0  # 64 keys: one chunk, nothing to join
    good = dict(q=FAKE, k=FAKE, v=FAKE, table=FAKE, seq=FAKE, start=FAKE, mask=FAKE, o=FAKE, lse=None, ws=FAKE, n=bytes_needed)

    def call(shape=s, cache=c, **kw):
        a = dict(good, **kw)
        return L.sp_cache_attn(ctypes.byref(shape), None if cache is None else ctypes.byref(cache), a["q"], a["k"], a["v"], a["table"],
                               a["seq"], a["start"], a["mask"], a["o"], a["lse"], a["ws"], a["n"], None)

    _said(call(cache=None), "SP_ERR_INVALID_ARG", b"cache is NULL")
    _said(L.sp_cache_attn(None, ctypes.byref(c), *[FAKE] * 10, bytes_needed, None), "SP_ERR_INVALID_ARG", b"shape is NULL")
    for x, name in (("q", b"q"), ("k", b"k_cache"), ("v", b"v_cache"), ("table", b"block_table"), ("seq", b"seq_len"),
                    ("start", b"tok_start"), ("mask", b"tree_mask"), ("o", b"o")):
        _said(call(**{x: None}), "SP_ERR_INVALID_ARG", name + b" is NULL")
        _said(call(**{x: FAKE + 2}), "SP_ERR_INVALID_ARG", name + b" is not")
    _said(call(lse=FAKE + 2), "SP_ERR_INVALID_ARG", b"lse")
    _said(call(shape=_step(max_pages=400, mask_words=0)), "SP_ERR_INVALID_ARG", b"go together")
    _said(call(ws=None), "SP_ERR_WORKSPACE", b"NULL")
    _said(call(ws=FAKE + 16), "SP_ERR_WORKSPACE", b"256-byte")
    _said(call(n=bytes_needed - 1), "SP_ERR_WORKSPACE", b"too small")
    # no tokens or no requests: done, and nothing is looked at
    for empty in (dict(n_tokens=0), dict(n_requests=0)):
        _said(L.sp_cache_attn(ctypes.byref(_step(**empty)), ctypes.byref(c), *[None] * 10, 0, None), "SP_OK")
    with pytest.raises(sp.SpError):
        sp.sp_cache_attn_workspace_bytes(_step(mask_words=9), c)


@pytest.mark.parametrize("bad,status,text", [
    (dict(n_tokens=-1), "SP_ERR_INVALID_ARG", b"negative"), (dict(head_dim=80), "SP_ERR_UNSUPPORTED", b"head_dim"),
    (dict(n_kv_heads=3), "SP_ERR_INVALID_ARG", b"n_q_heads"), (dict(rotary_dim=12), "SP_ERR_INVALID_ARG", b"rotary_dim"),
    (dict(rotary_dim=72), "SP_ERR_INVALID_ARG", b"rotary_dim"), (dict(rotary_dim=-8), "SP_ERR_INVALID_ARG", b"rotary_dim"),
    (dict(eps=-1.0), "SP_ERR_INVALID_ARG", b"eps"), (dict(eps=float("nan")), "SP_ERR_INVALID_ARG", b"eps"),
    (dict(q_stride_t=63), "SP_ERR_INVALID_ARG", b"q_stride_t"), (dict(k_stride_h=8), "SP_ERR_INVALID_ARG", b"k_stride_h"),
    (dict(v_stride_t=4), "SP_ERR_INVALID_ARG", b"v_stride_t"), (dict(qo_stride_h=0), "SP_ERR_INVALID_ARG", b"qo_stride_h"),
    (dict(ko_stride_t=-64), "SP_ERR_INVALID_ARG", b"ko_stride_t"),
])
def test_rope_geometry(bad, status, text):
    rc = sp.lib().sp_qk_norm_rope(ctypes.byref(_rope(**bad)), *[FAKE] * 9, ctypes.byref(_cache()), FAKE, FAKE, FAKE, None)
    _said(rc, status, text)


def test_rope_arguments():
    L = sp.lib()
    names = ["q", "k", "v", "q_weight", "k_weight", "inv_freq", "positions", "q_out", "k_out", "k_cache", "v_cache", "slots"]

    def call(shape=None, cache=True, **kw):
        a = {n: kw.get(n, FAKE) for n in names}
        return L.sp_qk_norm_rope(ctypes.byref(shape or _rope()), *[a[n] for n in names[:9]], ctypes.byref(_cache()) if cache else None,
                                 *[a[n] for n in names[9:]], None)

    for n in ("q", "k", "v", "inv_freq", "positions", "q_out", "k_cache", "v_cache", "slots"):
        _said(call(**{n: None}), "SP_ERR_INVALID_ARG", n.encode() + b" is NULL")
    for n in names:
        _said(call(**{n: FAKE + 2}), "SP_ERR_INVALID_ARG", n.encode() + b" is not")
    _said(call(cache=False, k_out=None), "SP_ERR_INVALID_ARG", b"go nowhere")
    _said(L.sp_qk_norm_rope(None, *[FAKE] * 9, None, FAKE, FAKE, FAKE, None), "SP_ERR_INVALID_ARG", b"shape is NULL")
    c = _cache(n_kv_heads=1)
    rc = L.sp_qk_norm_rope(ctypes.byref(_rope()), *[FAKE] * 9, ctypes.byref(c), FAKE, FAKE, FAKE, None)
    _said(rc, "SP_ERR_INVALID_ARG", b"the cache has")
    _said(L.sp_qk_norm_rope(ctypes.byref(_rope(n_tokens=0)), *[None] * 8, FAKE, None, None, None, None, None), "SP_OK")


def test_plan_arguments():
    L = sp.lib()
    names = ["ctx_len", "new_len", "n_held", "block_table", "free_pages", "free_capacity", "n_free", "parents", "mask_words",
             "n_held_out", "n_free_out", "tok_start", "seq_len", "positions", "slots", "status", "tree_mask", "workspace"]
    base = dict({n: FAKE + 512 * a for a, n in enumerate(names)}, free_capacity=8, mask_words=1)

    def call(n=3, tokens=10, page=16, width=4, ws=1 << 20, **kw):
        a = dict(base, **kw)
        return L.sp_cache_plan(n, tokens, page, width, *[a[x] for x in names], ws, None)

    pointers = [x for x in names if x not in ("free_capacity", "mask_words", "workspace")]
    for x in pointers:
        if x not in ("parents", "tree_mask"):
            _said(call(**{x: None}), "SP_ERR_INVALID_ARG", x.encode() + b" is NULL")
        _said(call(**{x: base[x] + 2}), "SP_ERR_INVALID_ARG", x.encode() + b" is not")
    _said(call(tree_mask=None), "SP_ERR_INVALID_ARG", b"go together")
    _said(call(mask_words=0), "SP_ERR_INVALID_ARG", b"go together")
    _said(call(mask_words=5), "SP_ERR_UNSUPPORTED", b"mask_words")
    _said(call(page=24), "SP_ERR_UNSUPPORTED", b"page_size")
    _said(call(n=-1), "SP_ERR_INVALID_ARG", b"negative")
    _said(call(tokens=-1), "SP_ERR_INVALID_ARG", b"negative")
    _said(call(tokens=(1 << 28) + 1), "SP_ERR_UNSUPPORTED", b"2^28")
    _said(call(width=0), "SP_ERR_INVALID_ARG", b"max_pages")
    _said(call(width=1 << 27), "SP_ERR_UNSUPPORTED", b"longer")
    _said(call(free_capacity=-1), "SP_ERR_INVALID_ARG", b"free_capacity")
    _said(call(seq_len=base["ctx_len"]), "SP_ERR_INVALID_ARG", b"seq_len")
    _said(call(workspace=None), "SP_ERR_WORKSPACE", b"NULL")
    _said(call(workspace=base["workspace"] + 4), "SP_ERR_WORKSPACE", b"256-byte")
    _said(call(ws=27), "SP_ERR_WORKSPACE", b"too small")
    assert sp.sp_cache_plan_workspace_bytes(3) == 28
    with pytest.raises(sp.SpError):
        sp.sp_cache_plan_workspace_bytes(-1)


def test_accept_arguments():
    L, c = sp.lib(), _cache()
    names = ["k_cache", "v_cache", "block_table", "ctx_len", "seq_len", "path", "n_accepted", "ctx_out"]

    def call(n=2, layers=3, stride=8 * 16 * 128, width=4, most=5, **kw):
        a = {x: kw.get(x, FAKE + 512 * b) for b, x in enumerate(names)}
        return L.sp_cache_accept(ctypes.byref(c), layers, stride, a["k_cache"], a["v_cache"], n, width, a["block_table"], a["ctx_len"],
                                 a["seq_len"], most, a["path"], a["n_accepted"], a["ctx_out"], None)

    for x in names:
        if x != "ctx_out":
            _said(call(**{x: None}), "SP_ERR_INVALID_ARG", x.encode() + b" is NULL")
        _said(call(**{x: FAKE + 2}), "SP_ERR_INVALID_ARG", x.encode() + b" is not")
    _said(call(n=-1), "SP_ERR_INVALID_ARG", b"negative")
    _said(call(layers=0), "SP_ERR_INVALID_ARG", b"n_layers")
    _said(call(width=0), "SP_ERR_INVALID_ARG", b"max_pages")
    _said(call(most=257), "SP_ERR_UNSUPPORTED", b"max_accept")
    _said(call(stride=12), "SP_ERR_INVALID_ARG", b"stride_layer")
    _said(call(ctx_out=FAKE + 512 * 3), "SP_ERR_INVALID_ARG", b"ctx_out")
    _said(call(n=0, **{x: None for x in names}), "SP_OK")


@pytest.mark.parametrize("where", ["block_table", "ctx_len", "seq_len", "path", "n_accepted"])
def test_accept_does_not_write_what_it_reads(where):
    """Workgroups of one request (layers, pieces of a row) read these while the first of them writes ctx_out."""
    L, c, at = sp.lib(), _cache(), dict(block_table=2, ctx_len=3, seq_len=4, path=5, n_accepted=6)
    a = [FAKE + 512 * i for i in range(8)]
    rc = L.sp_cache_accept(ctypes.byref(c), 3, 8 * 16 * 128, a[0], a[1], 2, 4, a[2], a[3], a[4], 5, a[5], a[6], a[at[where]], None)
    _said(rc, "SP_ERR_INVALID_ARG", b"ctx_out")


def test_binding_refuses_host_memory_and_other_sizes():
    """The binding looks at the tensors before the library sees an address: a host tensor's would fault the device."""
    import torch
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q, cache = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    c = sp.cache_shape_of(cache)
    assert (c.n_pages, c.page_size, c.n_kv_heads, c.head_dim, c.stride_page, c.stride_token, c.stride_head) == (3, 16, 2, 64, 2048, 128, 64)
    s = sp.step_shape_of(q, q, i32(2, 3), 1)
    assert (s.n_requests, s.n_tokens, s.n_q_heads, s.max_pages) == (2, 2, 4, 3)
    ws = torch.zeros(256, dtype=torch.uint8)
    with pytest.raises(ValueError, match="on cpu"):
        sp.sp_cache_attn(s, c, q, cache, cache, i32(2, 3), i32(2), i32(3), None, q, None, ws)
    r = sp.rope_shape_of(q, k, k, q, k, 64)
    with pytest.raises(ValueError, match="on cpu"):
        sp.sp_qk_norm_rope(r, q, k, k, None, None, torch.zeros(32), i32(2), q, k, c, cache, cache, i32(2))
    with pytest.raises(ValueError, match="needs inv_freq"):
        sp.sp_qk_norm_rope(r, q, k, k, None, None, None, i32(2), q, k)
    with pytest.raises(ValueError, match="needs v, k_cache"):
        sp.sp_qk_norm_rope(r, q, k, None, None, None, torch.zeros(32), i32(2), q, k, c, cache, cache, i32(2))
    with pytest.raises(ValueError, match="on cpu"):
        sp.sp_cache_plan(i32(2), i32(2), i32(2), i32(2, 3), i32(4), i32(1), 16, None, i32(2), i32(1), i32(3), i32(2), i32(5), i32(5),
                         i32(2), None, ws)
    with pytest.raises(ValueError, match="on cpu"):
        sp.sp_cache_accept(c, cache, cache, i32(2, 3), i32(2), i32(2), i32(2, 4), i32(2))
    with pytest.raises(ValueError, match="words a token"):
        sp.sp_cache_attn(s, c, q, cache, cache, i32(2, 3), i32(2), i32(3), torch.zeros(2, 1, dtype=torch.int64), q, None, ws)
    with pytest.raises(ValueError, match="one geometry"):
        sp.sp_cache_accept(c, cache, cache[None], i32(2, 3), i32(2), i32(2), i32(2, 4), i32(2))
