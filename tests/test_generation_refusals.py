"""What the calls on a paged cache refuse, without a GPU: the checks come before anything is enqueued."""
import ctypes

import numpy as np
import pytest

from oracle import generation_oracle as O


@pytest.fixture(scope="module")
def B():
    from paper_2607_25291_b200 import binding, build
    build.build()
    binding.library()
    return binding


ONE = ctypes.c_void_p(256)      # never dereferenced


def cache(B, **kw):
    c = B.CosaCacheStruct(k=256, v=256, k_bounds=256, page_table=256, k_scale=256, v_scale=256, table_stride=10, num_pages=100, page_size=16, hkv=2,
                          d=128, dtype=B.COSA_BF16, cache_dtype=B.COSA_BF16)
    for key, val in kw.items():
        setattr(c, key, (ctypes.c_int64 * 3)(*val) if key == "strides" else val)
    return c


BAD_CACHES = [
    ({"d": 96}, -2), ({"d": 256}, -2), ({"dtype": 2}, -2), ({"dtype": 7}, -2), ({"cache_dtype": 1}, -2), ({"hkv": 0}, -1), ({"page_size": 12}, -1),
    ({"page_size": 4}, -1), ({"page_size": 131072}, -1), ({"num_pages": 0}, -1), ({"num_pages": 2 ** 28}, -2), ({"table_stride": 0}, -1),
    ({"table_stride": 2 ** 28}, -2), ({"k": None}, -1), ({"v": 264}, -1), ({"cache_dtype": 2, "k_scale": None}, -1), ({"strides": (4096, 2048, 100)}, -1),
    ({"strides": (4096, 2048, 132)}, -1), ({"strides": (4096, 0, 128)}, -1), ({"strides": (0, 2048, 128)}, -1),
    ({"cache_dtype": 2, "strides": (4096, 2048, 136)}, -1), ({"k_bounds": 264}, -1)]


@pytest.mark.parametrize("bad,want", BAD_CACHES)
def test_caches(B, bad, want):
    L, c = B.library(), ctypes.byref(cache(B, **bad))
    assert L.cosa_cache_append(c, ONE, ONE, ONE, 1, None) == want
    assert L.cosa_decode_attention(c, ONE, 1, 8, ONE, None, None, 0, ONE, None, None) == want


def test_calls(B):
    L, c = B.library(), ctypes.byref(cache(B))
    assert L.cosa_cache_append(None, ONE, ONE, ONE, 1, None) == -1
    assert L.cosa_cache_append(c, None, ONE, ONE, 1, None) == -1
    assert L.cosa_cache_append(c, ONE, ctypes.c_void_p(260), ONE, 1, None) == -1
    assert L.cosa_cache_append(c, ONE, ONE, None, 1, None) == -1
    assert L.cosa_cache_append(c, ONE, ONE, ONE, -1, None) == -1
    assert L.cosa_cache_append(c, None, None, None, 0, None) == 0      # nothing to do
    opt = B.decode_options()
    opt.new_strides = (ctypes.c_int64 * 2)(300, 128)
    assert L.cosa_cache_append_ex(c, ONE, ONE, ONE, 2, None, ctypes.byref(opt)) == -1
    attend = lambda opt=None, q=ONE, batch=1, hq=8, lens=ONE, pages=None, count=None, pitch=0, out=ONE: L.cosa_decode_attention_ex(  # noqa: E731
        c, q, batch, hq, lens, pages, count, pitch, out, None, None, ctypes.byref(opt) if opt is not None else None)
    assert attend(q=None) == -1 and attend(lens=None) == -1 and attend(out=None) == -1
    assert attend(batch=0) == -1 and attend(hq=7) == -1 and attend(hq=0) == -1 and attend(batch=70000) == -2
    assert attend(q=ctypes.c_void_p(264)) == -1 and attend(out=ctypes.c_void_p(264)) == -1
    assert attend(pages=ONE) == -1 and attend(pages=ONE, count=ONE, pitch=0) == -1
    assert attend(B.decode_options(window=-1)) == -1 and attend(B.decode_options(ctas=-2)) == -1
    assert attend(B.decode_options(softmax_scale=-1.0)) == -1 and attend(B.decode_options(softmax_scale=float("nan"))) == -1
    assert attend(B.decode_options(impl=2)) == -2
    assert attend(pages=ONE, count=ONE, pitch=1 << 30) == -2      # more boxes than 32 bits count
    big = ctypes.byref(cache(B, table_stride=1 << 26, hkv=1))      # 2^30 tokens a request: more tiles than 32 bits count over 512 query heads
    assert L.cosa_decode_attention(big, ONE, 1, 512, ONE, None, None, 0, ONE, None, None) == -2
    assert L.cosa_decode_select(big, ONE, 1, 64, ONE, 0.5, ONE, ONE, 1 << 26, None) == -2
    opt = B.decode_options()
    opt.q_strides = (ctypes.c_int64 * 2)(1024, 100)
    assert attend(opt) == -1
    opt = B.decode_options()
    opt.out_strides = (ctypes.c_int64 * 2)(64, 128)
    assert attend(opt, batch=2) == -1
    select = lambda opt=None, budget=0.5, pitch=10, pages=ONE, count=ONE, c=c: L.cosa_decode_select_ex(  # noqa: E731
        c, ONE, 1, 8, ONE, budget, pages, count, pitch, None, ctypes.byref(opt) if opt is not None else None)
    assert select(budget=0.0) == -1 and select(budget=1.5) == -1 and select(budget=float("nan")) == -1
    assert select(pitch=4) == -1 and select(B.decode_options(min_pages=6), pitch=5) == -1 and select(B.decode_options(keep_first=3, keep_last=4), pitch=6) == -1
    assert select(pages=None) == -1 and select(count=None) == -1
    assert select(B.decode_options(keep_first=-1)) == -1 and select(B.decode_options(min_pages=-1)) == -1
    assert select(c=ctypes.byref(cache(B, k_bounds=None))) == -1


def test_workspaces_that_are_too_small(B):
    L, c = B.library(), cache(B, table_stride=200000)      # (short rows of the table need none)
    need = B.library().cosa_decode_workspace_bytes(0, ctypes.byref(c), 3, 8, None)
    assert need > 0
    opt = B.decode_options(workspace=256, workspace_bytes=need - 1)
    assert L.cosa_decode_select_ex(ctypes.byref(c), ONE, 3, 8, ONE, 0.5, ONE, ONE, 100000, None, ctypes.byref(opt)) == -3
    opt = B.decode_options(workspace=264, workspace_bytes=need)
    assert L.cosa_decode_select_ex(ctypes.byref(c), ONE, 3, 8, ONE, 0.5, ONE, ONE, 100000, None, ctypes.byref(opt)) == -3


def test_page_plans(B):
    L = B.library()
    p = lambda x: ctypes.c_void_p(x)  # noqa: E731

    def plan(lens=256, grow=512, batch=4, page=16, table=1024, width=8, ring=2048, pages=50, state=4096, out_lens=5120, out_state=6144, starts=7168,
             slots=8192, space=9):
        return L.cosa_page_plan(p(lens), p(grow), batch, page, p(table), width, p(ring), pages, p(state), p(out_lens), p(out_state), p(starts), p(slots),
                                None, None, space, None)

    for name in ("lens", "grow", "table", "ring", "state", "out_lens", "out_state", "starts", "slots"):
        assert plan(**{name: None}) == -1, name
    assert plan(batch=0) == -1 and plan(space=-1) == -1 and plan(page=10) == -1 and plan(width=0) == -1 and plan(pages=0) == -1
    assert plan(batch=8193) == -2 and plan(pages=2 ** 28) == -2
    assert plan(out_lens=256) == -1 and plan(out_state=4096) == -1 and plan(starts=512) == -1      # outputs over inputs


def test_oracle_by_hand():
    """The oracle itself, on cases small enough to be worked out."""
    got = O.page_plan([3, 8], [2, 1], 4, np.array([[5, -1, -1], [1, 2, -1]]), np.array([9, 7, 0, 0]), 0, 2, 4)
    assert got["lens"].tolist() == [5, 9] and got["table"].tolist() == [[5, 9, -1], [1, 2, 7]] and got["slots"].tolist() == [23, 36, 28, -1]
    assert got["starts"].tolist() == [0, 2, 3] and got["state"].tolist() == [2, 2] and got["positions"].tolist() == [3, 4, 8, -1]
    q, low, high = np.array([[1.0, -2.0] + [0.0] * 62]), np.zeros((3, 64)), np.zeros((3, 64))
    low[:, :2], high[:, :2] = [[0, 0], [-1, -3], [1, 1]], [[1, 1], [0, 4], [2, 2]]
    assert O.page_scores(q, low, high).tolist() == [[1.0, 6.0, 0.0]]
    assert O.select(q, low, high, 0.3).tolist() == [1] and O.select(q, low, high, 0.5, last=1).tolist() == [1, 2]
    out, lse, _ = O.attention(np.array([[1.0, 0.0]]), np.array([[0.0, 5.0], [np.log(3.0), 1.0]]), np.array([[4.0, 0.0], [0.0, 8.0]]), 1.0)
    assert np.allclose(out, [[1.0, 6.0]]) and np.allclose(lse, np.log(4.0))
    assert O.kept_tokens(10, 4, [2, 0, 7, -1]).tolist() == [8, 9, 0, 1, 2, 3] and O.kept_tokens(10, 4, None, 3).tolist() == [7, 8, 9]


def test_binding_refusals(B):
    import torch
    t = torch.zeros(2, 2, 16, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.make_cache(t, t, torch.zeros(1, 2, dtype=torch.int32))      # not on the GPU
    with pytest.raises(ValueError):
        B.make_cache(None, None, torch.zeros(1, 2, dtype=torch.int32))      # neither pools nor bounds


class OnGpu:
    """A CPU tensor that says it is on the GPU, for checks that come before any use of its memory."""

    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


class NoCalls:
    """Stands for the library where nothing may reach it."""

    def __getattr__(self, name):
        def called(*args):
            raise AssertionError(f"{name} was called")
        return called


def test_expanded_tensors_are_refused(B, monkeypatch):
    """A tensor that repeats its elements (a stride of zero) is not handed on: the C calls would take it for a dense one and read, or write, past its end."""
    import torch
    monkeypatch.setattr(B, "_lib", NoCalls())
    monkeypatch.setattr(B, "_stream_ptr", lambda stream: 0)
    bf16, i32, d = torch.bfloat16, torch.int32, 128
    new = lambda *shape, dtype=bf16: OnGpu(torch.zeros(*shape, dtype=dtype))      # noqa: E731
    row, heads, tokens = (OnGpu(torch.zeros(*shape, dtype=bf16).expand(3, 4, d)) for shape in ((1, 1, d), (1, 4, d), (3, 1, d)))
    table, lens, slots = new(3, 10, dtype=i32), new(3, dtype=i32), new(3, dtype=i32)
    pool = new(5, 4, 16, d)
    cache = B.make_cache(pool, pool, table, bounds=new(5, 4, 2, d))
    pages, count = new(3, 4, 10, dtype=i32), new(3, 4, dtype=i32)
    for bad in (row, heads, tokens):
        for call in (lambda: B.cosa_decode_attention(cache, bad, lens, new(3, 4, d)), lambda: B.cosa_decode_attention(cache, new(3, 4, d), lens, bad),
                     lambda: B.cosa_cache_append(cache, bad, bad, slots), lambda: B.cosa_decode_select(cache, bad, lens, 0.5, pages, count)):
            with pytest.raises(ValueError):
                call()
    for shape in ((1, 1, 1, d), (5, 1, 1, d), (1, 4, 16, d), (5, 4, 1, d)):
        bad = OnGpu(torch.zeros(*shape, dtype=bf16).expand(5, 4, 16, d))
        with pytest.raises(ValueError):
            B.make_cache(bad, bad, table)
    # a dimension of one element may have any stride
    one = torch.zeros(3, 8, d, dtype=bf16)[:, ::8].as_strided((3, 1, d), (8 * d, 0, 1))
    assert B._rows(OnGpu(one), one.shape, "q")[1] == (8 * d, 0)


def test_expanded_tensors_of_a_prompt_are_refused(B, monkeypatch):
    """The same for the calls on a prompt, whose strides of zero stand for the dense layout too."""
    import torch
    monkeypatch.setattr(B, "_lib", NoCalls())
    monkeypatch.setattr(B, "_set_strides", lambda opt, **kw: None)
    monkeypatch.setattr(B, "_stream_ptr", lambda stream: 0)
    new = lambda *shape, dtype=torch.bfloat16: OnGpu(torch.zeros(*shape, dtype=dtype))      # noqa: E731
    lists = new(1, 4, 2, 2, dtype=torch.int32), new(1, 4, 2, dtype=torch.int32)
    q, k, out = new(1, 4, 256, 128), new(1, 2, 256, 128), new(1, 4, 256, 128)
    for heads, slot in ((4, 0), (2, 1), (4, 3)):
        bad = OnGpu(torch.zeros(1, 1, 1, 128, dtype=torch.bfloat16).expand(1, heads, 256, 128).as_strided((1, heads, 256, 128), (0, 0, 0, 1)))
        args = [q, k, k, out]
        args[slot] = bad
        if slot == 1:
            args[2] = bad
        with pytest.raises(ValueError):
            B.cosa_osk_attention(args[0], args[1], args[2], *lists, 1.0, args[3])
        if slot < 2:
            with pytest.raises(ValueError):
                B.cosa_kap_select(args[0], args[1], 0.5, *lists)


def test_oracle_of_infinite_scores_by_hand():
    """A page of infinite score holds its head's maximum; a head that knows only -inf, and a score that is no number, have no say."""
    inf, q = np.inf, np.array([[1.0, 0.0] + [0.0] * 62, [0.0, -1.0] + [0.0] * 62])
    low, high = np.zeros((4, 64)), np.zeros((4, 64))
    low[:, 0], high[:, 0] = -1.0, [1.0, 2.0, inf, 3.0]
    low[:, 1], high[:, 1] = [-5.0, -1.0, -1.0, -2.0], 0.0
    assert O.page_scores(q, low, high).tolist() == [[1.0, 2.0, inf, 3.0], [5.0, 1.0, 1.0, 2.0]]
    assert O.select(q, low, high, 0.25).tolist() == [0] and O.select(q, low, high, 0.5).tolist() == [0, 2] and O.select(q, low, high, 0.75).tolist() == [0, 2, 3]
    q[1, 0] = 0.5
    low[:, 0], high[:, 0] = [-1.0, -1.0, -inf, -1.0], [-1.0, -1.0, -inf, -1.0]
    assert O.select(q, low, high, 0.5).tolist() == [0, 1]      # the first head has its maximum in pages 0, 1 and 3, the second in page 0
    low[:, 0], high[:, 0] = -inf, -inf
    assert O.select(q, low, high, 0.5).tolist() == [0, 1]      # nobody has a say: the lowest indices
    low[0, 0], high[0, 0] = inf, -inf      # (the bounds of a page whose keys are all NaN in this channel)
    assert O.page_scores(q, low, high)[0].tolist() == [inf, -inf, -inf, -inf]


def test_misaligned_words(B):
    """Pointers to 32- and 64-bit words that are no multiples of their size."""
    L, off, q = B.library(), ctypes.c_void_p(258), ctypes.c_void_p(4096)
    for bad in ({"page_table": 258}, {"k_scale": 257, "cache_dtype": B.COSA_E4M3}, {"v_scale": 258, "cache_dtype": B.COSA_E4M3}):
        c = ctypes.byref(cache(B, **bad))
        assert L.cosa_cache_append(c, ONE, ONE, ONE, 1, None) == -1
        assert L.cosa_decode_attention(c, ONE, 1, 8, ONE, None, None, 0, ONE, None, None) == -1
    c = ctypes.byref(cache(B))
    for at in range(4):
        lens, pages, count, lse = (off if i == at else ONE for i in range(4))
        assert L.cosa_decode_attention(c, ONE, 1, 8, lens, pages, count, 4, ONE, lse, None) == -1
        if at < 3:
            assert L.cosa_decode_select(c, ONE, 1, 8, lens, 0.5, pages, count, 10, None) == -1
    good = [256, 512, 4, 16, 1024, 8, 2048, 50, 4096, 5120, 6144, 7168, 8192, 9216, 10240, 9]
    for i in (0, 1, 4, 6, 8, 9, 10, 11, 12, 13, 14):
        for step in ((2, 4) if i in (8, 10) else (1, 2)):
            args = [x + step if j == i else x for j, x in enumerate(good)]
            assert L.cosa_page_plan(*(ctypes.c_void_p(x) if x > 200 else x for x in args), None) == -1, i


def test_the_example_uses_what_a_user_has():
    """Its prompt goes from the cache's pools through the binding's public calls."""
    import inspect
    import re
    from paper_2607_25291_b200 import generate
    assert not re.search(r"cosa\._|library\(|byref", inspect.getsource(generate))


@pytest.mark.parametrize("args", [["--tokens", "1"], ["--prompts", "200"], ["--prompts", "256,0"], ["--page", "48"], ["--page", "256", "--prompts", "384"],
                                  ["--budget", "0"], ["--budget", "1.5"]])
def test_the_example_refuses(args, monkeypatch, capsys):
    from paper_2607_25291_b200 import generate
    monkeypatch.setattr("sys.argv", ["generate", *args])
    with pytest.raises(SystemExit) as e:
        generate.main()
    assert e.value.code == 2 and "error" in capsys.readouterr().err
