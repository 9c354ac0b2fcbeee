"""What the calls refuse before anything is launched: shapes, types, devices, numbers out of their ranges."""
import ctypes as C

import pytest
import torch

from paper_2511_21699_b200 import _lib, api
from tests.operator_refs import context

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _t(*shape, dtype=torch.int32, device="cuda"):
    return torch.zeros(*shape, dtype=dtype, device=device)


@pytest.fixture()
def cb():
    return context(batch=2, n_q_heads=4, n_kv_heads=2, head_dim=64, max_nodes=8)


def _refused(call, good, wrong, launches):
    """Each of the wrong values in its place is refused and nothing is launched; then the good ones are not."""
    for name, values in wrong.items():
        for v in values:
            before = launches()
            with pytest.raises((api.CachebackError, TypeError)):
                call(**{**good, name: v})
            assert launches() == before, (name, v)
    call(**good)
    torch.cuda.synchronize()


def test_pages_assign(cb):
    good = dict(want_len=_t(2), block_table=_t(2, 9), held=_t(2), free_pages=_t(18), n_free=_t(1))
    f, cpu = torch.float32, _t(2, device="cpu")
    _refused(cb.cb_pages_assign, good, dict(want_len=[cpu, _t(3), _t(2, dtype=torch.int64), None], block_table=[_t(2), _t(3, 9), _t(9, 2).t(), _t(2, 0)], held=[_t(1), _t(2, dtype=f)],
                                            free_pages=[_t(2, 9), _t(0), _t(18, dtype=torch.int64)], n_free=[_t(2), _t(0)]), cb.launch_count)


def test_slot_map(cb):
    new = lambda n: dict(slots=_t(n, dtype=torch.int64), positions=_t(n), seqs=_t(n))
    good = dict(q_start=_t(3), ctx_len=_t(2), block_table=_t(2, 9), num_pages=18, n_rows=5, res=new(5))
    _refused(cb.cb_slot_map, good, dict(q_start=[_t(2)], ctx_len=[_t(3)], block_table=[_t(1, 9)], num_pages=[0, -1, 1 << 31], n_rows=[-1, 4, 1 << 31],
                                        res=[new(4), dict(new(5), slots=_t(5)), dict(new(5), seqs=_t(5, dtype=torch.int64))]), cb.launch_count)
    assert {k: v.numel() for k, v in cb.cb_slot_map(_t(3), _t(2), _t(2, 9), 18, 0).items()} == dict(slots=0, positions=0, seqs=0)


def test_block_summary(cb):
    good = dict(k_pool=_t(18, 16, 2, 64, dtype=BF), block_table=_t(2, 9), from_len=_t(2), to_len=_t(2), k_mean=_t(18, 2, 64, dtype=torch.int8), k_scale=_t(18, 2, dtype=torch.float32), block=64)
    _refused(cb.cb_block_summary, good, dict(k_pool=[_t(18, 16, 4, 64, dtype=BF), _t(18, 16, 2, 64, dtype=torch.float16), _t(17, 16, 2, 64, dtype=BF), _t(18, 8, 2, 64, dtype=BF)],
                                             from_len=[_t(3)], to_len=[_t(1)], k_mean=[_t(18, 2, 64, dtype=torch.uint8), _t(18, 2, 32, dtype=torch.int8)], k_scale=[_t(17, 2, dtype=torch.float32)],
                                             block=[0, 8, 48, 65, 256, -16, 1 << 40]), cb.launch_count)
    assert [x.shape for x in cb.alloc_summary(7)] == [(7, 2, 64), (7, 2)]


def _select_args(**kw):
    return {**dict(q=_t(5, 4, 64, dtype=BF), k_mean=_t(18, 2, 64, dtype=torch.int8), k_scale=_t(18, 2, dtype=torch.float32), block_table=_t(2, 9), ctx_len=_t(2), q_start=_t(3), block=64,
                   n_select=4, n_first=1, n_last=2, blocks=_t(2, 2, 4)), **kw}


def test_block_select(cb):
    wrong = dict(q=[_t(5, 2, 64, dtype=BF), _t(5, 4, 64, dtype=torch.float32), _t(5, 4, 128, dtype=BF), _t(4, 64, dtype=BF), _t(5, 8, 64, dtype=BF)[:, ::2]],
                 k_mean=[_t(18, 2, 64, dtype=torch.uint8), _t(18, 1, 64, dtype=torch.int8)], k_scale=[_t(18, 2, dtype=BF), _t(18, 3, dtype=torch.float32)], block_table=[_t(3, 9)],
                 ctx_len=[_t(1)], q_start=[_t(2), None], n_nodes=[_t(2)], block=[15, 0, 512], n_select=[0, 3, 5, -1], n_first=[-1, 3], n_last=[0, -1, 4], blocks=[_t(2, 4, 4), _t(2, 2, 4, dtype=torch.int64)],
                 max_chunk=[-1], max_ctx=[-1])
    _refused(cb.cb_block_select, _select_args(), wrong, cb.launch_count)
    _refused(cb.cb_block_select, _select_args(q=_t(2, 8, 4, 64, dtype=BF), q_start=None, n_nodes=_t(2)), dict(q=[_t(5, 4, 64, dtype=BF), _t(2, 7, 4, 64, dtype=BF)], n_nodes=[_t(3), None]), cb.launch_count)
    with pytest.raises(api.CachebackError):                                  # more than 1,024 a list
        cb.cb_block_select(**_select_args(n_select=1025, blocks=_t(2, 2, 1025)))
    cb.cb_block_select(**_select_args(n_select=1024, blocks=_t(2, 2, 1024)))
    wide = _t(2, 16385)                                                      # a bound of more than 16,384 blocks
    with pytest.raises(api.CachebackError, match="unsupported"):
        cb.cb_block_select(**_select_args(block=16, block_table=wide))
    cb.cb_block_select(**_select_args(block=16, block_table=wide, max_ctx=16 * 16384))
    assert cb.cb_poll_status()[0] == 0


def test_block_attn(cb):
    pool = lambda **k: _t(18, 16, k.get("h", 2), 64, dtype=BF)
    good = dict(q=_t(5, 4, 64, dtype=BF), k_pool=pool(), v_pool=pool(), block_table=_t(2, 9), q_start=_t(3), ctx_len=_t(2), blocks=_t(2, 2, 4), block=64)
    _refused(cb.cb_block_attn, good, dict(q=[_t(5, 2, 64, dtype=BF), _t(5, 4, 64)], k_pool=[pool(h=4)], v_pool=[pool(h=1), _t(17, 16, 2, 64, dtype=BF)], blocks=[_t(2, 4, 4), _t(2, 2), _t(2, 2, 0), _t(2, 2, 1025)],
                                          block=[16 * 3, 0, 256], out=[_t(5, 4, 32, dtype=BF), good["q"]], lse=[_t(5, 4), _t(4, 5, dtype=torch.float32)], max_chunk=[-1], max_ctx=[-5],
                                          scale=[-1.0, float("nan"), float("inf")]), cb.launch_count)
    assert cb.cb_block_attn(**dict(good, q=_t(0, 4, 64, dtype=BF))).shape == (0, 4, 64)


def test_block_tree_attn(cb):
    pool, node = _t(18, 16, 2, 64, dtype=BF), lambda h: _t(2, 8, h, 64, dtype=BF)
    good = dict(q=node(4), k_pool=pool, v_pool=pool, block_table=_t(2, 9), ctx_len=_t(2), k_tree=node(2), v_tree=node(2), tree_mask=_t(2, 8, 1), n_nodes=_t(2), blocks=_t(2, 2, 4), block=64)
    _refused(cb.cb_block_tree_attn, good, dict(q=[node(2), _t(16, 4, 64, dtype=BF)], k_tree=[node(4)], v_tree=[_t(2, 7, 2, 64, dtype=BF)], tree_mask=[_t(2, 8, 2), _t(2, 8, 1, dtype=torch.float32)], n_nodes=[_t(3)],
                                               blocks=[_t(1, 2, 4), _t(2, 2, 0)], block=[63], out=[node(2), good["q"]], lse=[_t(2, 8, 4, dtype=torch.float32)], max_ctx=[-1], scale=[-0.5, float("nan")]),
             cb.launch_count)


def test_misaligned_pointers(cb):
    lib = _lib.load()
    base = _t(1 << 20, dtype=torch.uint8).data_ptr()
    a = _lib.CbBlockSummaryArgsC(base + 2, base, base, base, base, base, 9, 18, 64)
    assert lib.cb_block_summary(cb._h, C.byref(a), None) == _lib.CB_ERR_INVALID_ARG
    a = _lib.CbBlockSummaryArgsC(base, base, base, base, base + 4, base, 9, 18, 64)
    assert lib.cb_block_summary(cb._h, C.byref(a), None) == _lib.CB_ERR_INVALID_ARG
    s = _lib.CbBlockSelectArgsC(base + 8, base, None, base, base, base, base, base, 5, 9, 18, 64, 4, 1, 1, 0, 0)
    assert lib.cb_block_select(cb._h, C.byref(s), None) == _lib.CB_ERR_INVALID_ARG
    for null in ("k_mean", "block_table", "ctx_len", "blocks"):
        s = _lib.CbBlockSelectArgsC(base, base, None, base, base, base, base, base, 5, 9, 18, 64, 4, 1, 1, 0, 0)
        setattr(s, null, None)
        assert lib.cb_block_select(cb._h, C.byref(s), None) == _lib.CB_ERR_INVALID_ARG


def test_numbers_above_what_is_counted(cb):
    """Sums of pages and of blocks are counted below 2^30; what could exceed that is refused by its size alone, before anything is read."""
    lib = _lib.load()
    base = _t(1 << 10, dtype=torch.uint8).data_ptr()
    unsupported = 6                                                          # CB_ERR_UNSUPPORTED
    before = cb.launch_count()
    assert lib.cb_pages_assign(cb._h, base, base, 9, base, base, 1 << 30, base, None) == unsupported
    for block, most in ((16, 1 << 29), (64, (1 << 31) - 1)):                # (2 sequences of 2^29 blocks; 2^31 - 1 pages are 2^29 blocks)
        a = _lib.CbBlockSummaryArgsC(base, base, base, base, base, base, most, 18, block)
        assert lib.cb_block_summary(cb._h, C.byref(a), None) == unsupported
    assert cb.launch_count() == before
