"""Memory that a call would write over while it reads it, or that is not its to
write, is refused: the C ABI, on addresses that are never dereferenced."""
import pytest

from paper_2504_11320_amd import binding as B
from paper_2504_11320_amd import kv
from test_kv_more_host import batch, cache, eviction, norm, rows, turn

AT = 1 << 44   # memory of every argument, far from the others'
K, V, KS, VS, Q, OUT, LSE, W, TABLE, LENS, KEPT, LEFT, WS, TO, SLOTS = (AT + (i << 32) for i in range(15))


def eight(**kw):
    return cache(**{**dict(k=K, v=V, k_scale=KS, v_scale=VS, type=kv.INT8), **kw})


def sixteen(**kw):
    return cache(**{**dict(k=K, v=V), **kw})


def refused(rc, what="overlap"):
    assert rc == B.WS_EINVAL
    assert what in kv._lib().wait_sim_last_error().decode()


# a cache of 4 pages of 16 rows of 2 heads of 64: 128 rows, 16-bit ones of 128 bytes
ROWS, ROW8, ROW16 = 128, 64, 128


def weigh(c, w=W, ws=None, bytes_=0, **kw):
    b = dict(table=TABLE, starts=LENS + 4096, kv_lens=LENS)
    return kv._lib().wait_kv_weigh(c, batch(**{**b, **kw}), rows(data=Q, token=256), LSE, w, 1, ws, bytes_,
                                   None)


@pytest.mark.parametrize("w", [K, K + ROWS * ROW8 - 4, V, V + ROWS * ROW8 - 4, KS, VS, VS + 4 * ROWS - 4,
                               VS - 4 * ROWS + 4, Q, Q + 3 * 512 + 4 * 128 - 4, LSE, LSE + 4 * 4 * 4 - 4, TABLE,
                               TABLE + 4 * 15, LENS, LENS + 4, LENS + 4096])
def test_weights_that_lie_in_something_else(w):
    refused(weigh(eight(), w=w))
    if not KS - 4096 <= w < VS + 4096:
        refused(weigh(sixteen(), w=w))


def test_a_workspace_that_lies_in_something_else():
    """Weighing: rows that are split need one."""
    many = dict(n_tokens=512, max_q_len=512, max_kv_len=128)
    assert weigh(eight(), **many) == B.WS_EWORKSPACE
    for ws in (K, V, KS, VS, Q, LSE, W, W + 4 * ROWS - 4, TABLE, LENS):
        refused(weigh(eight(), ws=ws, bytes_=1 << 26, **many), "workspace")
    long = dict(table_cols=1 << 10, table_stride=1 << 10, max_kv_len=10000)
    assert evict(eight(), **long) == B.WS_EWORKSPACE
    for ws in (K, V, KS, VS, W, TABLE, LENS, KEPT, LEFT):
        refused(evict(eight(), ws=ws, bytes_=1 << 26, **long), "workspace")


def evict(c, w=W, kept=KEPT, left=LEFT, ws=None, bytes_=0, **kw):
    e = dict(table=TABLE, kv_lens=LENS)
    return kv._lib().wait_kv_evict(c, eviction(**{**e, **kw}), w, kept, left, ws, bytes_, None)


@pytest.mark.parametrize("to", [0, TO])
def test_an_eviction_into_its_own_arguments(to):
    kw = dict(to=to)
    for w in (K, V, KS, VS, VS + 4 * ROWS - 4, TABLE, LENS):
        refused(evict(eight(), w=w, **kw))
    for at in (K, V + ROWS * ROW8 - 4, KS, VS, W, W + 4 * ROWS - 4, TABLE, LENS):
        refused(evict(eight(), kept=at, **kw))
        if at != LENS:
            refused(evict(eight(), left=at, **kw))
    refused(evict(eight(), left=LENS + 4, **kw), "memory of their own")
    refused(evict(eight(), left=KEPT + 4 * 2 * 2 * 20 - 4, **kw))
    refused(evict(eight(k=TABLE), **kw))
    refused(evict(sixteen(v=LENS), **kw))
    if to:
        refused(evict(eight(), w=TO, **kw))
        refused(evict(eight(), kept=TO + 4 * 3, **kw))


def test_keys_and_values_of_one_place():
    """Rows that move within their pages go there once."""
    refused(evict(sixteen(v=K)))
    refused(evict(sixteen(v=K + ROWS * ROW16 - 16)))
    refused(evict(eight(v_scale=KS)))


def test_an_eviction_to_the_requests_own_pages():
    """Rows on their way to other pages do not wait for one another."""
    refused(evict(sixteen(), to=TABLE), "own pages")
    refused(evict(sixteen(), to=TABLE, to_stride=8, to_cols=8), "own pages")


def test_queries_that_enter_the_cache():
    q, k, v = (rows(data=Q + 128 * i, token=512) for i in (0, 4, 6))

    def enter(out, c):
        return kv._lib().wait_kv_enter(c, q, rows(data=out, token=256), 4, k, v, SLOTS, 3, norm(), norm(), turn(),
                                       None)

    for c, row in ((eight(), ROW8), (sixteen(), ROW16)):
        for at in (K, K + ROWS * row - 2, K - 3 * 512 + 2, V, V + ROWS * row - 2):
            refused(enter(at, c))
    for at in (KS, VS, VS + 4 * ROWS - 2):
        refused(enter(at, eight()))
