"""Host side of the paged cache's operators, on the CPU: libwisv.so runs in a child process on a stand-in for the HIP runtime
(stub_hip.c: kernels are logged, not run).  Every refusal comes before a launch, with a message; good calls launch what they
should; the oracle itself is pinned to hand-worked numbers."""
import subprocess
import sys
import textwrap

import numpy as np
import pytest
import torch

from oracle import paged as ref
from paper_2604_17701_amd import binding
from test_host_failures import PRELUDE, ROOT, stub  # noqa: F401

PAGED = '''
buf = np.zeros(1 << 16, np.float32)
P = (buf.ctypes.data + 15) // 16 * 16
h = create(configs.TINY, 1, 64, 4)
stub.stub_log_clear()


def text():
    return lib.wisv_last_error(h).decode()


def plan(**kw):
    d = dict(batch=2, page_size=16, max_pages=4, n_free=3, max_tokens=9, cached_len=P, new_len=P, free_pages=P, block_table=P, q_start=P,
             kv_len=P, positions=P, slots=P, n_used=P, status=P)
    return lib.wisv_paged_plan(h, C.byref(B.wisv_paged_plan_args(**{**d, **kw})))


def append(**kw):
    d = dict(n_tokens=5, n_heads=4, n_kv_heads=2, head_dim=64, dtype=1, page_size=16, n_pages=3, n_rope=8, q=P, k=P, v=P, q_out=P + 4096,
             q_stride=256, k_stride=128, v_stride=128, q_out_stride=256, positions=P, slots=P, cos=P, sin=P, k_pages=P, v_pages=P)
    return lib.wisv_paged_append(h, C.byref(B.wisv_paged_append_args(**{**d, **kw})))


def attn_args(**kw):
    d = dict(batch=2, n_tokens=5, n_heads=4, n_kv_heads=2, head_dim=64, dtype=1, page_size=16, n_pages=3, max_pages=2, q=P, out=P,
             q_stride=256, out_stride=256, k_pages=P, v_pages=P, block_table=P, q_start=P, kv_len=P)
    return B.wisv_paged_attention_args(**{**d, **kw})


def need(**kw):
    n = C.c_size_t(77)
    assert lib.wisv_paged_attention_workspace(h, C.byref(attn_args(**kw)), C.byref(n)) == 0, text()
    return n.value


def attn(**kw):
    return lib.wisv_paged_attention(h, C.byref(attn_args(**kw)))

'''


def run(stub, body):
    code = f"ROOT, STUB = {ROOT!r}, {stub!r}\n" + PRELUDE + PAGED + textwrap.dedent(body) + "\nprint('done')\n"
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("done"), r.stdout + r.stderr


def test_plan_refuses_bad_arguments(stub):
    run(stub, '''
        assert plan() == 0 and len(log()) == 1, (text(), log())
        stub.stub_log_clear()
        for kw, what in ((dict(batch=0), "batch"), (dict(batch=4097), "batch"), (dict(page_size=8), "page_size"), (dict(page_size=48), "page_size"),
                         (dict(page_size=8192), "page_size"), (dict(max_pages=0), "max_pages"), (dict(max_pages=1 << 28), "max_pages"), (dict(n_free=-1), "n_free"),
                         (dict(free_pages=None), "free_pages"), (dict(max_tokens=0), "max_tokens"), (dict(cached_len=None), "NULL"),
                         (dict(status=None), "NULL"), (dict(slots=None), "NULL")):
            assert plan(**kw) == B.WISV_EINVAL and what in text(), (kw, text())
        assert lib.wisv_paged_plan(h, None) == B.WISV_EINVAL and lib.wisv_paged_plan(None, None) == B.WISV_EINVAL
        assert log() == []
        assert plan(n_free=0, free_pages=None) == 0
    ''')


def test_append_refuses_bad_arguments(stub):
    run(stub, '''
        assert append() == 0 and len(log()) == 1, (text(), log())
        stub.stub_log_clear()
        for kw, what in ((dict(n_tokens=-1), "n_tokens"), (dict(head_dim=96), "head_dim"), (dict(dtype=2), "dtype"), (dict(page_size=24), "page_size"),
                         (dict(n_pages=0), "n_pages"), (dict(n_pages=1 << 28), "n_pages"), (dict(k_pages=None), "pool"), (dict(v_pages=P + 2), "16 bytes"),
                         (dict(page_stride=100), "page_stride"), (dict(page_stride=2052), "page_stride"), (dict(n_heads=-1), "n_heads"), (dict(cos=None), "cos"),
                         (dict(n_rope=0), "rotary"), (dict(sin=P + 4), "rotary"), (dict(slots=None), "NULL"), (dict(positions=None), "NULL"),
                         (dict(q=None), "q, k, v"), (dict(k=None), "q, k, v"), (dict(v=P + 8), "q, k, v"), (dict(q_stride=252), "q, k, v"),
                         (dict(k_stride=132), "q, k, v"), (dict(v_stride=64), "q, k, v"), (dict(q_out=P, q_out_stride=512), "another stride"),
                         (dict(n_kv_heads=0), "n_kv_heads")):
            assert append(**kw) == B.WISV_EINVAL and what in text(), (kw, text())
        assert append(n_tokens=2**31 - 1, n_heads=65536, q_stride=1 << 22, q_out_stride=1 << 22) == B.WISV_EUNSUPPORTED
        assert append(n_tokens=0, slots=None, q=None) == 0       # nothing to do
        assert lib.wisv_paged_append(h, None) == B.WISV_EINVAL and lib.wisv_paged_append(None, None) == B.WISV_EINVAL
        assert log() == []
        assert append(n_heads=0, q=None, q_out=None, cos=None, sin=None, positions=None) == 0 and len(log()) == 1
        assert append(q_out=P) == 0 and append(dtype=0, q_stride=260, k_stride=132) == 0
    ''')


def test_attention_refuses_bad_arguments(stub):
    run(stub, '''
        assert need() == 0 and attn() == 0 and log(), text()
        stub.stub_log_clear()
        for kw, what in ((dict(batch=-1), "batch"), (dict(n_tokens=-1), "n_tokens"), (dict(n_heads=3), "n_heads"), (dict(n_heads=0), "n_heads"),
                         (dict(n_kv_heads=0), "n_kv_heads"), (dict(head_dim=80), "head_dim"), (dict(dtype=-1), "dtype"), (dict(page_size=100), "page_size"),
                         (dict(max_pages=0), "max_pages"), (dict(max_pages=2**31 - 1), "max_pages"), (dict(max_new=-1), "max_new"), (dict(max_len=-1), "max_len"),
                         (dict(window=-1), "window"), (dict(softcap=-1.0), "softcap"), (dict(softcap=float("nan")), "softcap"),
                         (dict(softcap=float("inf")), "softcap"), (dict(scale=float("inf")), "scale"), (dict(q=None), "q and out"), (dict(out=P + 4), "q and out"),
                         (dict(q_stride=128), "q and out"), (dict(out_stride=257), "q and out"), (dict(block_table=None), "NULL"), (dict(q_start=None), "NULL"),
                         (dict(kv_len=None), "NULL"), (dict(page_stride=8), "page_stride")):
            assert attn(**kw) == B.WISV_EINVAL and what in text(), (kw, text())
            n = C.c_size_t()
            assert lib.wisv_paged_attention_workspace(h, C.byref(attn_args(**kw)), C.byref(n)) == B.WISV_EINVAL
        big = 2**31 - 1
        assert attn(n_tokens=big) == B.WISV_EUNSUPPORTED
        assert lib.wisv_paged_attention(h, None) == B.WISV_EINVAL and lib.wisv_paged_attention(None, None) == B.WISV_EINVAL
        assert lib.wisv_paged_attention_workspace(h, C.byref(attn_args()), None) == B.WISV_EINVAL
        assert attn(batch=0, q=None) == 0 and attn(n_tokens=0, block_table=None) == 0     # nothing to do
        # a cache that is worth cutting needs room for its parts
        long = dict(batch=1, n_tokens=1, max_pages=4096, max_len=65536, max_new=1)
        n = need(**long)
        assert n > 0
        for kw in (dict(), dict(workspace=P, workspace_bytes=n - 1), dict(workspace=P + 4, workspace_bytes=n), dict(workspace_bytes=n)):
            assert attn(**long, **kw) == B.WISV_EINVAL and "workspace" in text(), kw
        assert log() == []
        assert attn(**long, workspace=P, workspace_bytes=n) == 0 and any("join" in l for l in log())
    ''')


def test_struct_sizes_match_the_header_layout():
    import ctypes as C
    assert C.sizeof(binding.wisv_paged_plan_args) == 5 * 4 + 4 + 11 * 8
    assert C.sizeof(binding.wisv_paged_append_args) == 8 * 4 + 4 * 8 + 4 * 8 + 6 * 8 + 2 * 8
    assert C.sizeof(binding.wisv_paged_attention_args) == 14 * 4 + 4 * 8 + 3 * 8 + 6 * 8 + 2 * 8


def test_paged_fill_follows_the_documented_layout():
    kp, vp = binding.new_paged_cache(5, 2, 16, 32, torch.float32, "cpu")
    k, v = torch.randn(2, 37, 32), torch.randn(2, 37, 32)
    binding.paged_fill(kp, vp, [4, 0, 2], k, v)
    for pos in (0, 7, 8, 15, 16, 31, 36):
        page = [4, 0, 2][pos // 16]
        for d in (0, 5, 31):
            flat = vp[page, 1].reshape(-1)
            assert kp[page, 1, pos % 16, d] == k[1, pos, d] and flat[((pos % 16) // 8 * 32 + d) * 8 + pos % 8] == v[1, pos, d]
    assert float(kp[1].abs().sum() + kp[3].abs().sum() + kp[2, :, 5:].abs().sum()) == 0.0
    gk, gv, there = ref.gather(kp.double().numpy(), vp.double().numpy(), [4, 0, 2], 37)
    assert there.all() and np.array_equal(gk, k.double().numpy()) and np.array_equal(gv, v.double().numpy())


def test_oracle_plan_by_hand():
    # 3 of a page's 4 positions held, 2 more: one new page; idle; 8 held in a full table row: refused; 5 new: two pages
    got = ref.plan([3, 0, 8, 0], [2, 0, 1, 5], [9, 8, 7], [[5, -1], [-1, -1], [1, 2], [-1, -1]], 4, 9)
    q_start, kv_len, positions, slots, used, status, table = got
    assert q_start.tolist() == [0, 2, 2, 3, 8] and kv_len.tolist() == [5, 0, 8, 5]
    assert positions.tolist() == [3, 4, 8, 0, 1, 2, 3, 4, 0]
    assert slots[:2].tolist() == [5 * 4 + 3, 9 * 4] and slots[2] == -1            # the third request's row is full
    assert status.tolist() == [0, 0, 2, 0] and table[3].tolist() == [8, 7] and used.tolist() == [3]
    assert slots[3:8].tolist() == [32, 33, 34, 35, 28] and slots[8] == -1


def test_oracle_attention_by_hand():
    """Two keys with scores 0 and ln 3: weights 1/4 and 3/4; a window of one, a cap, a bias and a prefix change them as written."""
    kp, vp = np.zeros((1, 1, 16, 2)), np.zeros((1, 1, 2, 2, 8))
    kp[0, 0, 1] = [np.log(3.0), 0.0]
    vp[0, 0, 0, :, 0], vp[0, 0, 0, :, 1] = [4.0, 0.0], [0.0, 4.0]
    q = np.array([[[1.0, 0.0]]])
    call = lambda **kw: ref.attention(q, kp, vp, [[0]], [0, 1], [2], scale=1.0, **kw)[0][0, 0].tolist()  # noqa: E731
    assert np.allclose(call(), [1.0, 3.0])
    assert np.allclose(call(window=1), [0.0, 4.0])
    assert np.allclose(call(window=1, prefix=[1]), [1.0, 3.0])
    cap = 2 * np.tanh(np.log(3.0) / 2)                                            # = 1
    assert np.allclose(cap, 1.0) and np.allclose(call(softcap=2.0), [4 / (1 + np.e), 4 * np.e / (1 + np.e)])
    assert np.allclose(call(slopes=[np.log(3.0)]), [0.4, 3.6])                    # the nearer key gains another factor of 3
    out = ref.attention(np.ones((3, 1, 2)), kp, vp, [[0]], [0, 3], [2], scale=1.0)[0]
    assert (out[0] == 0).all() and np.allclose(out[1, 0], [4.0, 0.0])             # the first row lies before the cache


def test_calls_that_one_launch_does_not_cover_are_refused(stub):
    run(stub, '''
        assert attn(n_tokens=1 << 25, n_heads=4) == B.WISV_EUNSUPPORTED and "2^26" in text()
        assert attn(batch=1 << 20, n_kv_heads=2) == B.WISV_EUNSUPPORTED and "2^21" in text()
        assert attn(max_pages=1 << 27) == B.WISV_EINVAL and "2^30" in text()
        for cap in (1e-37, 16385.0, float("inf"), float("nan"), -2.0):
            assert attn(softcap=cap) == B.WISV_EINVAL and "softcap" in text(), cap
        assert append(n_tokens=1 << 30) == B.WISV_EUNSUPPORTED and "one launch" in text()
        assert log() == []
        assert attn(n_tokens=1 << 24, n_heads=4, max_new=8, max_pages=2) == 0 and attn(window=2**31 - 1) == 0
    ''')


def test_a_device_that_refuses_the_lds_is_an_error(stub):
    """A prompt's kernel wants 64 KB of LDS or more: a device that refuses says so before anything is enqueued, and the next
    call is not blamed for it."""
    run(stub, '''
        many = dict(n_tokens=100, max_new=90)
        stub.stub_refuse_lds(1)
        assert attn(**many) == B.WISV_EHIP and "LDS" in text() and log() == []
        assert attn() == 0 and len(log()) == 1            # few rows need no such kernel
        stub.stub_refuse_lds(0)
        stub.stub_log_clear()
        assert attn(**many) == 0 and any("prompt" in l for l in log()), (text(), log())
    ''')


def test_which_kernel_serves_which_rows(stub):
    run(stub, '''
        def served(**kw):
            stub.stub_log_clear()
            need_ = need(**kw)
            assert attn(**kw, workspace=P if need_ else None, workspace_bytes=need_) == 0, text()
            return "".join("p" if "prompt" in l else "j" if "join" in l else "r" if "rows" in l else "?" for l in log())
        assert served(max_new=5, n_tokens=10) == "r" and served(max_new=5, n_tokens=10, dtype=0) == "r"
        assert served(max_new=17, n_tokens=20) == "p" and served(max_new=17, n_tokens=20, dtype=0) == "r"    # 34 rows per KV head
        wide = dict(head_dim=128, q_stride=512, out_stride=512)
        assert served(max_new=8, n_tokens=8, **wide) == "r" and served(max_new=9, n_tokens=9, **wide) == "p"
        long = dict(batch=1, max_pages=4096, max_len=65536)
        assert served(n_tokens=1, max_new=1, **long) == "rj" and served(n_tokens=40, max_new=40, **long) == "pj"
    ''')


def test_which_kernel_serves_float_prompts(stub):
    run(stub, '''
        def served(**kw):
            stub.stub_log_clear()
            need_ = need(dtype=0, **kw)
            assert attn(dtype=0, **kw, workspace=P if need_ else None, workspace_bytes=need_) == 0, text()
            return "".join("p" if "prompt" in l else "j" if "join" in l else "r" if "rows" in l else "?" for l in log())
        # two rows per token, two KV heads: 128 tiles from 4096 tokens on
        assert served(n_tokens=4096, max_new=2048) == "p" and served(n_tokens=4032, max_new=2048) == "r"
        for batch, kernel in ((64, "p"), (85, "p"), (90, "r")):     # 128, 97 and 92 of a tile's rows
            assert served(n_tokens=4096 if batch == 64 else 48 * 85 + 49 if batch == 85 else 46 * 90, max_new=64, batch=batch) == kernel, batch
        assert served(n_tokens=4096, max_new=2048, head_dim=32, q_stride=128, out_stride=128) == "r"
        assert served(n_tokens=4096, max_new=2048, head_dim=256, q_stride=1024, out_stride=1024) == "p"
        stub.stub_refuse_lds(1)
        assert attn(dtype=0, n_tokens=4096, max_new=2048, head_dim=128, q_stride=512, out_stride=512) == B.WISV_EHIP and "LDS" in text()
        stub.stub_refuse_lds(0)
    ''')


class OnHost:
    """Stands for a ctx whose tensors lie on the host (get_device() -1): the binding's checks alone."""
    device = type("Device", (), {"index": -1})()

    def __getattr__(self, name):
        return getattr(binding.Context, name).__get__(self)


def test_the_binding_refuses_pools_whose_pages_overlap():
    k, v = binding.new_paged_cache(1, 2, 16, 64, torch.float32, "cpu")
    spread = binding.new_paged_cache(3, 4, 16, 64, torch.float32, "cpu")
    assert OnHost()._pools(k, v) == (1, 2, 16, 64, binding.WISV_F32, 2 * 16 * 64)
    assert OnHost()._pools(spread[0][:, :2], spread[1][:, :2]) == (3, 2, 16, 64, binding.WISV_F32, 4 * 16 * 64)
    one = (k.expand(3, -1, -1, -1), v.expand(3, -1, -1, -1, -1))       # one page three times: no distance, which would mean the usual one
    near = (spread[0].as_strided((3, 2, 16, 64), (1024, 1024, 64, 1)), spread[1].as_strided((3, 2, 2, 64, 8), (1024, 1024, 512, 8, 1)))
    for pools in (one, near):
        with pytest.raises(ValueError, match="distance"):
            OnHost()._pools(*pools)


def test_the_binding_refuses_numbers_that_would_wrap():
    k, v = binding.new_paged_cache(2, 1, 16, 32, torch.float32, "cpu")
    ints = torch.zeros(1, dtype=torch.int32)
    q, table = torch.zeros(1, 1, 32), torch.zeros((1, 2), dtype=torch.int32)
    for kw, what in ((dict(window=1 << 32), "window"), (dict(window=-(1 << 32)), "window"), (dict(max_new=1 << 31), "max_new"), (dict(max_len=1 << 31), "max_len"),
                     (dict(scale=1e-50), "scale"), (dict(scale=-1e-50), "scale"), (dict(softcap=1e-50), "softcap")):
        with pytest.raises(ValueError, match=what):
            OnHost().wisv_paged_attention(q, k, v, table, torch.zeros(2, dtype=torch.int32), ints, **kw)
    for kw in (dict(page_size=16, max_tokens=0), dict(page_size=16, max_tokens=1 << 32), dict(page_size=(1 << 32) + 16, max_tokens=4)):
        with pytest.raises(ValueError, match="max_tokens"):
            OnHost().wisv_paged_plan(ints, ints, ints, table, **kw)


def test_filling_needs_pages_for_every_position():
    k, v = binding.new_paged_cache(4, 1, 16, 32, torch.float32, "cpu")
    rows = torch.randn(1, 33, 32)
    with pytest.raises(ValueError, match="hold"):
        binding.paged_fill(k, v, [2, 0], rows, rows)
    assert not k.any() and not v.any()
    binding.paged_fill(k, v, [2, 0, 3], rows, rows)
    assert torch.equal(torch.cat([k[2], k[0], k[3]], 1)[:, :33], rows)


def test_a_plan_over_its_own_lengths_is_one_workgroups(stub):
    """Workgroups read the lengths apart from each other: where one of the outputs lies over them, a single one does the work."""
    run(stub, '''
        Q = lambda i: P + 4096 * i
        apart = dict(cached_len=Q(0), new_len=Q(1), free_pages=Q(2), block_table=Q(3), q_start=Q(4), kv_len=Q(5), positions=Q(6), slots=Q(7), n_used=Q(8),
                     status=Q(9))

        def threads(**kw):
            stub.stub_log_clear()
            assert plan(**{**apart, **kw}) == 0 and len(log()) == 1, (text(), log())
            return [n for n in (256, 1024) if f"ILi{n}E" in log()[0]]
        assert threads() == [256]
        for out in ("q_start", "kv_len", "positions", "slots", "n_used", "status", "block_table"):
            for i in (0, 1):
                assert threads(**{out: Q(i)}) == [1024] and threads(**{out: Q(i) + 4}) == [1024], (out, i)
        # two requests' lengths are eight bytes: what lies beside them does not touch them
        assert threads(kv_len=Q(0) + 8) == [256] and threads(kv_len=Q(1) - 8) == [256] and threads(kv_len=Q(1) - 4) == [1024]
        assert threads(q_start=Q(1) - 12) == [256] and threads(q_start=Q(1) - 8) == [1024]
    ''')


@pytest.mark.parametrize("i", range(6))
def test_the_binding_refuses_plans_whose_outputs_overlap(i):
    b, tokens = 3, 10
    lens, free, table = torch.zeros(b, dtype=torch.int32), torch.arange(12, dtype=torch.int32), torch.zeros((b, 4), dtype=torch.int32)
    sizes = (b + 1, b, tokens, tokens, 1, b)
    shared = torch.zeros(64, dtype=torch.int32)
    for other in (free, table.view(-1), None):
        out = [torch.zeros(n, dtype=torch.int32) for n in sizes]
        if other is None:     # the last of one output is the first of the next
            out[i], out[(i + 1) % 6] = shared[:sizes[i]], shared[sizes[i] - 1:][:sizes[(i + 1) % 6]]
        else:
            out[i] = other[12 - sizes[i]:]
        with pytest.raises(ValueError, match="overlap"):
            OnHost().wisv_paged_plan(lens, lens, free, table, 16, tokens, out=binding.PagePlan(*out))


def test_which_rows_meet():
    """Against the bytes themselves."""
    import itertools
    for p, s, w, q, t, v, n in itertools.product((0, 3, 8), (4, 8, 9), (1, 4), (0, 1, 5, 12, 30), (4, 8), (2, 4), (1, 2, 3)):
        a, b = ({x + i * y + j for i in range(n) for j in range(z)} for x, y, z in ((p, s, w), (q, t, v)))
        got = binding._rows_meet(p, s, w, q, t, v, n)
        assert got or not a & b
        assert not got or a & b or s != t, (p, s, w, q, t, v, n)


def test_the_binding_refuses_results_over_what_a_call_reads():
    h, g, hd, n = 4, 2, 32, 6
    buf = torch.zeros((40, h + 2 * g + 2, hd))
    q, k, v = buf[4:4 + n, :h], buf[4:4 + n, h:h + g], buf[4:4 + n, h + g:h + 2 * g]
    pools = torch.zeros((2, 3, g, 16, hd))
    kp, vp = pools[0], pools[1].view(3, g, 2, hd, 8)
    ints = torch.zeros(n, dtype=torch.int32)
    lens, starts, table = torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros((1, 2), dtype=torch.int32)
    one = buf.view(-1)
    over = {"a head further": buf[4:4 + n, 1:1 + h], "a row further": buf[5:5 + n, :h], "from the keys on": buf[4:4 + n, h - 1:2 * h - 1], "another stride":
            one[4 * buf.stride(0):].as_strided((n, h, hd), (h * hd, hd, 1)), "the keys' pool": pools.view(-1)[64:].as_strided((n, h, hd), (h * hd, hd, 1)),
            "the values' pool": pools.view(-1)[pools[0].numel() + 512:].as_strided((n, h, hd), (h * hd, hd, 1))}
    for what, out in over.items():
        with pytest.raises(ValueError, match="overlap"):
            OnHost().wisv_paged_append(q, k, v, None, ints, kp, vp, q_out=out)
        if what != "from the keys on":
            with pytest.raises(ValueError, match="overlap"):
                OnHost().wisv_paged_attention(q, kp, vp, table, starts, lens, out=out)
    with pytest.raises(ValueError, match="overlap"):
        OnHost().wisv_paged_append(q, buf[4:4 + n, h - 1:h + 1], v, None, ints, kp, vp, q_out=q)     # in place, over a head of the keys
    with pytest.raises(ValueError, match="overlap"):
        OnHost().wisv_paged_append(k, k, v, None, ints, kp, vp, q_out=k)
    with pytest.raises(ValueError, match="heads of q"):
        OnHost().wisv_paged_attention(q, kp, vp, table, starts, lens, out=torch.zeros((n, h + 1, hd)))
    result = lambda out: OnHost()._result("out", out, torch.float32, n, hd, h, ((q.data_ptr(), q.stride(0), h), (k.data_ptr(), k.stride(0), g)), (kp.data_ptr(), vp.data_ptr()), kp.numel())  # noqa: E731
    for out in (q, torch.zeros((n, h, hd)), buf[10:10 + n, :h], buf[4:4 + n, h + g:]):     # in place, elsewhere, rows behind, columns beside
        assert result(out) == (out.data_ptr(), out.stride(0))


def test_settings_beyond_the_arithmetic_are_refused(stub):
    """2 scale / (ln 2 softcap) beyond float would make the score of orthogonal vectors, 0, no number."""
    run(stub, '''
        for kw in (dict(scale=3e38), dict(scale=-2e38), dict(scale=1e9, softcap=1e-30), dict(scale=-1e9, softcap=1e-30), dict(scale=1e38, softcap=0.5)):
            assert np.isinf(np.float32(2.885390082) * np.float32(kw["scale"])) or np.isinf(np.float32(2.885390082) * np.float32(kw["scale"]) / np.float32(kw["softcap"]))
            assert attn(**kw) == B.WISV_EINVAL and "scale" in text(), kw
            n = C.c_size_t()
            assert lib.wisv_paged_attention_workspace(h, C.byref(attn_args(**kw)), C.byref(n)) == B.WISV_EINVAL
        assert log() == []
        for kw in (dict(scale=1e38), dict(scale=-1e38), dict(scale=1e8, softcap=1e-30), dict(scale=1e38, softcap=16384.0), dict(softcap=1e-30)):
            assert attn(**kw) == 0, (kw, text())
    ''')


def test_the_binding_refuses_rows_that_want_a_gradient():
    h, g, hd, n = 4, 2, 32, 6
    q, k, v = torch.zeros(n, h, hd), torch.zeros(n, g, hd), torch.zeros(n, g, hd)
    kp, vp = binding.new_paged_cache(3, g, 16, hd, torch.float32, "cpu")
    ints, lens, starts, table = (torch.zeros(m, dtype=torch.int32) for m in (n, 1, 2, 2))
    args = dict(block_table=table.view(1, 2), q_start=starts, kv_len=lens)
    want = lambda t: (t * 1.0).requires_grad_()  # noqa: E731
    for rows in ((want(q), k, v), (q, want(k), v), (q, k, want(v))):
        with pytest.raises(ValueError, match="gradient"):
            OnHost().wisv_paged_append(*rows, None, ints, kp, vp)
    for kw in (dict(q=want(q)), dict(q=q, out=want(q)), dict(q=want(q) * 2), dict(q=q, slopes=want(torch.zeros(h)))):
        with pytest.raises(ValueError, match="gradient"):
            OnHost().wisv_paged_attention(**{**dict(k_pages=kp, v_pages=vp, **args), **kw})
    for call in (lambda: OnHost()._rows("q", want(q).detach(), torch.float32, n, hd), torch.no_grad()(lambda: OnHost()._rows("q", want(q), torch.float32, n, hd))):
        assert call()[1:] == (h, h * hd)
