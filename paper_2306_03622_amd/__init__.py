"""Pipelined model swap-in and execution on one AMD MI355X (libtorpor + ctypes binding)."""
from .torpor import *  # noqa: F401,F403
from .serve import PagedCache, TPS_E4M3, tps_cache_append, tps_cache_attention, tps_cache_read, tps_lora  # noqa: F401
from .torpor import Runtime, ModelDesc, TorporError, HostArena, lib, host_lib  # noqa: F401
