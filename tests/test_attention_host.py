"""Host side of dc_kv_append and dc_attention_paged: what is refused before anything is enqueued (no GPU is touched: the addresses
are made up), what the workspace calls say, and pins of the oracle."""
import numpy as np
import pytest

import oracle.attention as oa
import paper_2502_15443_amd as dc

ADDR = 1 << 20
E_ARG, E_CAP = -1, -2


def cache(**kw):
    c = dc.KVCache(ADDR, ADDR, 10, 2, 128, 16, dc.TYPE_BF16)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def batch(**kw):
    b = dc.KVBatch(3, 20, 18, 100, ADDR, ADDR, 7, row_start_dev=ADDR)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def rows(**kw):
    s = (1024, 128)
    r = dc.KVRows(dc.TYPE_BF16, 4, ADDR, ADDR, ADDR, 2 * ADDR, rot_dim=64, cos_dev=ADDR, sin_dev=ADDR, n_positions=100, k_strides=s,
                  v_strides=s, q_strides=s, q_out_strides=s)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def attention(**kw):
    a = dc.Attention(4, ADDR, 2 * ADDR, None, 0.1, q_strides=(512, 128), out_strides=(512, 128))
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_CACHE = [dict(type=2), dict(n_kv_heads=0), dict(n_kv_heads=65536), dict(head_dim=0), dict(head_dim=96), dict(head_dim=512),
             dict(page_tokens=0), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=512), dict(n_pages=0), dict(n_pages=2 ** 31),
             dict(k_dev=None), dict(v_dev=None), dict(k_dev=ADDR + 8), dict(v_dev=ADDR + 2)]
BAD_BATCH = [dict(n_seqs=0), dict(n_seqs=65536), dict(n_rows=0), dict(n_rows=2 ** 31), dict(max_new=0), dict(max_new=21), dict(max_len=0),
             dict(pages_stride=0), dict(pages_stride=2 ** 27), dict(len_dev=None), dict(pages_dev=None), dict(row_start_dev=None),
             dict(prefix_len=5), dict(prefix_pages_dev=ADDR), dict(prefix_len=2 ** 31 - 112, prefix_pages_dev=ADDR)]
BAD_ROWS = [dict(type=3), dict(n_heads=65536), dict(rot_dim=8), dict(rot_dim=144), dict(pairing=2), dict(n_positions=0), dict(k_dev=None),
            dict(v_dev=None), dict(q_dev=None), dict(q_out_dev=None), dict(cos_dev=None), dict(sin_dev=None), dict(k_dev=ADDR + 4),
            dict(v_dev=ADDR + 4), dict(q_dev=ADDR + 4), dict(q_out_dev=ADDR + 4), dict(cos_dev=ADDR + 4), dict(sin_dev=ADDR + 4),
            dict(k_row_stride=1020), dict(k_head_stride=132), dict(v_row_stride=1), dict(v_head_stride=4), dict(q_row_stride=1030),
            dict(q_head_stride=127), dict(q_out_row_stride=500), dict(q_out_head_stride=64), dict(q_out_row_stride=256),
            dict(q_dev=2 * ADDR, type=dc.TYPE_F16), dict(q_dev=2 * ADDR, q_row_stride=2048), dict(q_dev=2 * ADDR, q_head_stride=136)]
BAD_ATTENTION = [dict(n_heads=0), dict(n_heads=3), dict(n_heads=65536), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_dev=None),
                 dict(out_dev=None), dict(out_dev=ADDR), dict(q_dev=ADDR + 8), dict(out_dev=ADDR + 8), dict(lse_dev=ADDR + 2),
                 dict(q_row_stride=4), dict(q_head_stride=4), dict(out_row_stride=4), dict(out_head_stride=4), dict(out_head_stride=64),
                 dict(out_row_stride=256), dict(out_row_stride=64, out_head_stride=2048)]


def refused(code, call, *args):
    with pytest.raises(dc.DCError) as e:
        call(*args)
    assert e.value.code == code


@pytest.mark.parametrize("bad", BAD_CACHE, ids=str)
def test_caches_that_are_refused(bad):
    refused(E_ARG, dc.kv_append, cache(**bad), batch(), rows())
    refused(E_ARG, dc.attention_paged_workspace, cache(**bad), batch(), attention())
    refused(E_ARG, dc.attention_paged, cache(**bad), batch(), attention(), ADDR, 1 << 40)


@pytest.mark.parametrize("bad", BAD_BATCH, ids=str)
def test_batches_that_are_refused(bad):
    refused(E_ARG, dc.kv_append, cache(), batch(**bad), rows())
    refused(E_ARG, dc.attention_paged_workspace, cache(), batch(**bad), attention())
    refused(E_ARG, dc.attention_paged, cache(), batch(**bad), attention(), ADDR, 1 << 40)


@pytest.mark.parametrize("bad", BAD_ROWS, ids=str)
def test_rows_that_are_refused(bad):
    refused(E_ARG, dc.kv_append, cache(), batch(), rows(**bad))


@pytest.mark.parametrize("bad", BAD_ATTENTION, ids=str)
def test_attentions_that_are_refused(bad):
    refused(E_ARG, dc.attention_paged_workspace, cache(), batch(), attention(**bad))
    refused(E_ARG, dc.attention_paged, cache(), batch(), attention(**bad), ADDR, 1 << 40)


def test_null_descriptions_are_refused():
    refused(E_ARG, dc.kv_append, None, batch(), rows())
    refused(E_ARG, dc.kv_append, cache(), None, rows())
    refused(E_ARG, dc.kv_append, cache(), batch(), None)
    refused(E_ARG, dc.attention_paged, None, batch(), attention(), ADDR, 1 << 40)
    refused(E_ARG, dc.attention_paged, cache(), None, attention(), ADDR, 1 << 40)
    refused(E_ARG, dc.attention_paged, cache(), batch(), None, ADDR, 1 << 40)


def test_strides_come_from_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros((5, 8, 128), dtype=torch.bfloat16)
    r = dc.KVRows(dc.TYPE_BF16, 4, x[:, 4:6], x[:, 6:], x[:, :4], torch.zeros((4, 5, 128), dtype=torch.bfloat16).transpose(0, 1))
    assert (r.k_row_stride, r.k_head_stride, r.q_row_stride, r.q_out_row_stride, r.q_out_head_stride) == (1024, 128, 1024, 128, 640)
    assert r.v_dev == x.data_ptr() + 6 * 128 * 2
    with pytest.raises(ValueError):
        dc.Attention(4, x.transpose(1, 2), x, None, 1.0)
    with pytest.raises(ValueError):
        dc.Attention(4, ADDR, x, None, 1.0)


def test_oracle_attention_by_hand():
    k = np.zeros((2, 1, 16, 64))
    v = np.zeros((2, 1, 16, 64))
    batch = {"lens": [3], "starts": [0, 2], "pages": np.array([[1]]), "prefix_len": 0, "prefix_pages": []}
    k[1, 0, :3, 0] = [np.log(2), np.log(3), np.log(5)]
    v[1, 0, :3, 0] = [1, 10, 100]
    q = np.zeros((2, 1, 64))
    q[:, 0, 0] = 1
    out, lse, _ = oa.attend(k, v, batch, q, 1.0)
    assert np.allclose(out[:, 0, 0], [32 / 5, 532 / 10]) and np.allclose(lse[:, 0], np.log([5, 10]))
    out, lse, _ = oa.attend(k, v, batch, q, 1.0, window=1, sinks=1)
    assert np.allclose(out[:, 0, 0], [32 / 5, 502 / 7]) and np.allclose(lse[:, 0], np.log([5, 7]))
    out, lse, _ = oa.attend(k, v, dict(batch, pages=np.array([[-1]])), q, 1.0)
    assert (out == 0).all() and np.isneginf(lse).all()


def test_oracle_attention_does_not_depend_on_how_tokens_are_held():
    r = np.random.default_rng(3)
    flat_k, flat_v = r.standard_normal((2, 50, 2, 64))
    q = r.standard_normal((4, 4, 64))
    results = []
    for page, prefix in ((16, 0), (32, 0), (16, 20), (16, 49)):
        n = 8
        k, v = np.full((2, n, 2, page, 64), np.nan)
        batch = {"lens": [50], "starts": [0, 4], "pages": np.array([[3, 5, 2, 7]]), "prefix_len": prefix, "prefix_pages": [6, 1, 4, 0]}
        for j in range(50):
            p, at = oa.place_of(batch, 0, j, page, n)
            k[p, :, at], v[p, :, at] = flat_k[j], flat_v[j]
        results.append(oa.attend(k, v, batch, q, 0.3, 30, 2)[:2])
    for out, lse in results[1:]:
        assert np.allclose(out, results[0][0], atol=1e-13) and np.allclose(lse, results[0][1], atol=1e-13)


def test_oracle_rotation():
    x = np.arange(8.0)[None] + 1
    cos, sin = np.cos([0.3, 1.1]), np.sin([0.3, 1.1])
    y = oa.rotate(x, cos, sin, False)
    assert np.allclose(y[0, 0] + 1j * y[0, 2], (1 + 3j) * np.exp(0.3j)) and np.allclose(y[0, 1] + 1j * y[0, 3], (2 + 4j) * np.exp(1.1j))
    y2 = oa.rotate(x, cos, sin, True)
    assert np.allclose(y2[0, 0] + 1j * y2[0, 1], (1 + 2j) * np.exp(0.3j)) and np.allclose(y2[0, 2] + 1j * y2[0, 3], (3 + 4j) * np.exp(1.1j))
    assert np.array_equal(y[0, 4:], x[0, 4:]) and np.array_equal(y2[0, 4:], x[0, 4:])
